// Token embedding: y[r] = scale * table[ids[r]], and the table's gradient by tokens sorted by id:
//   grad[v] (+)= scale * sum over the rows r with ids[r] = v of dy[r].
//
// The lookup is one pass bound by memory.  The gradient has three steps, none of which adds in an order that varies:
//   sort   (id, position) pairs by id, stable, in shared memory: a cluster of up to 8 CTAs holds up to 65 536 tokens and exchanges them by
//          distributed shared memory, so that a digit's pass costs two cluster barriers and no launch.  Digits are of up to 9 bits: two passes for
//          every vocabulary of less than 2^18.  The CTAs beside it write the zeros of a gradient that is not added to.  More tokens: a
//          cluster for each 65 536, and their sorted lists are merged, every pair finding its place by a search in the others.
//   runs   a block takes a stretch of the sorted tokens and 256 columns, its warps an eighth each, and adds the rows of every run of equal ids in
//          order of position.  Runs inside go to the gradient; what reaches over a warp's end is joined in the block, over the block's end left as a
//          partial row.
//   join   one warp per block end adds the partial rows of the run that crosses it.
// 16 384 tokens of a vocabulary of 32 000, 512 columns, bfloat16: sort 9 us (two passes of some 5000 cycles of latencies on 8 multiprocessors), runs 8, join 4; a micro-batch
// reads its gradient in 2.6 us at the memory's rate.  262 144 tokens, 128 000 x 2048: zeros, and the sort beside them, 178 us (6.0 TB/s), merge 11, runs 251 (5.5 TB/s
// of rows read and written), join 13: bound by memory.  One block a sort, as it began, took 6 ms for 16 384 tokens.
#include <cooperative_groups.h>

#include <algorithm>

#include "../../include/asteroid.h"
#include "common.cuh"
#include "kernels.h"

namespace ast {
namespace {

namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------ lookup
// Rows of whole 16-byte vectors: a thread's unit is 8 consecutive columns, a block's two a thread, some whole rows or a stretch of one; a unit's row is found by a
// multiplication (with the divisions that a flat index takes the pass was bound by its instructions, 65 us for 131 072 rows of 1024 columns; 60 so).
// Other rows: a warp takes 8 pieces a lane of one row, of 4, 2 or 1 columns as the addresses allow (131 072 rows of 1023 columns: 240 us with a thread a column
// and a row searched for each, 135 so).
constexpr int LOOKUP_UNITS = 2, LOOKUP_PIECES = 8;
constexpr unsigned LOOKUP_BLOCK = 256 * LOOKUP_UNITS;

template <int BYTES> struct Bits;
template <> struct Bits<2> {
    typedef unsigned short type;
};
template <> struct Bits<4> {
    typedef unsigned type;
};
template <> struct Bits<8> {
    typedef uint2 type;
};
template <> struct Bits<16> {
    typedef uint4 type;
};

template <typename S, int V> __device__ __forceinline__ void load_cols(const S* p, float* f) {
    if constexpr (V == 8) {
        constexpr int N = Vec<S>::N;
#pragma unroll
        for (int i = 0; i < V / N; ++i) {
            Vec<S> r;
            r.load(p, i);
            r.unpack(f + i * N);
        }
    } else {
        typedef typename Bits<V * sizeof(S)>::type B;
        B b = *reinterpret_cast<const B*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_f<S>(reinterpret_cast<const S*>(&b)[i]);
    }
}
template <typename T, int V> __device__ __forceinline__ void store_cols(T* p, const float* f) {
    if constexpr (V == 8) {
        constexpr int N = Vec<T>::N;
#pragma unroll
        for (int i = 0; i < V / N; ++i) {
            Vec<T> r;
            r.pack(f + i * N);
            r.store(p, i);
        }
    } else {
        typedef typename Bits<V * sizeof(T)>::type B;
        B b;
#pragma unroll
        for (int i = 0; i < V; ++i) reinterpret_cast<T*>(&b)[i] = from_f<T>(f[i]);
        *reinterpret_cast<B*>(p) = b;
    }
}

struct LookupShape {
    size_t rows, ldy;
    unsigned per_row, rows_per_block;            // units of a row; rows of a block
    unsigned inv;                                // 2^20 / units of a block's row, rounded up
    int vocab, dim;
    float scale;
};

template <typename S, typename T>
__global__ void __launch_bounds__(256) lookup_kernel(const S* __restrict__ table, const int32_t* __restrict__ ids, T* __restrict__ y, const LookupShape a) {
    pdl_wait();
    pdl_launch();
    constexpr int UNITS = LOOKUP_UNITS, V = 8;
    constexpr unsigned BLOCK = LOOKUP_BLOCK;
    const size_t row0 = (size_t)blockIdx.x * a.rows_per_block;
    const unsigned c0 = blockIdx.y * BLOCK, width = min(a.per_row - c0, BLOCK);
    float f[UNITS][V];
    size_t row[UNITS];
    unsigned c[UNITS];
    int id[UNITS];
    bool in[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const unsigned u = j * 256 + threadIdx.x, r = (u * a.inv) >> 20;         // u, the row's units <= 512: exact; 0 where a row has more
        row[j] = row0 + r;
        c[j] = (c0 + u - r * width) * V;
        in[j] = u < a.rows_per_block * width && row[j] < a.rows;
        id[j] = in[j] ? __ldg(ids + row[j]) : -1;
    }
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        if ((unsigned)id[j] < (unsigned)a.vocab) {
            load_cols<S, V>(table + (size_t)id[j] * a.dim + c[j], f[j]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) f[j][i] = 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        if (!in[j]) continue;
        const bool ok = (unsigned)id[j] < (unsigned)a.vocab;
#pragma unroll
        for (int i = 0; i < V; ++i) f[j][i] = ok ? f[j][i] * a.scale : 0.f;
        store_cols<T, V>(y + row[j] * a.ldy + c[j], f[j]);
    }
}

template <typename S, typename T, int V>
__global__ void __launch_bounds__(256) lookup_rows_kernel(const S* __restrict__ table, const int32_t* __restrict__ ids, T* __restrict__ y, const LookupShape a) {
    pdl_wait();
    pdl_launch();
    const size_t row = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    const int c0 = (int)blockIdx.y * (32 * V * LOOKUP_PIECES) + (threadIdx.x & 31) * V, id = __ldg(ids + row);
    const bool ok = (unsigned)id < (unsigned)a.vocab;
    const S* p = table + (size_t)(ok ? id : 0) * a.dim + c0;
    T* q = y + row * a.ldy + c0;
    float f[LOOKUP_PIECES][V];
#pragma unroll
    for (int j = 0; j < LOOKUP_PIECES; ++j)
        if (c0 + j * 32 * V < a.dim) load_cols<S, V>(p + j * 32 * V, f[j]);
#pragma unroll
    for (int j = 0; j < LOOKUP_PIECES; ++j) {
        if (c0 + j * 32 * V >= a.dim) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) f[j][i] = ok ? f[j][i] * a.scale : 0.f;
        store_cols<T, V>(q + j * 32 * V, f[j]);
    }
}

template <typename S, typename T> void launch_lookup(const void* table, const int32_t* ids, void* y, LookupShape a, cudaStream_t st) {
    const S* t = static_cast<const S*>(table);
    T* o = static_cast<T*>(y);
    const uintptr_t at = reinterpret_cast<uintptr_t>(table), to = reinterpret_cast<uintptr_t>(y);
    auto whole = [&](int v) { return a.dim % v == 0 && a.ldy % v == 0 && at % (v * sizeof(S)) == 0 && to % (v * sizeof(T)) == 0; };
    if (a.dim % 8 == 0 && a.ldy % (16 / sizeof(T)) == 0 && (at | to) % 16 == 0) {
        a.per_row = a.dim / 8;
        const unsigned width = std::min(a.per_row, LOOKUP_BLOCK);
        a.rows_per_block = LOOKUP_BLOCK / width;
        a.inv = ((1u << 20) + width - 1) / width;
        const dim3 blocks((unsigned)((a.rows + a.rows_per_block - 1) / a.rows_per_block), (a.per_row + LOOKUP_BLOCK - 1) / LOOKUP_BLOCK);
        launch_pdl(lookup_kernel<S, T>, blocks, 256, 0, st, t, ids, o, a);
        return;
    }
    const int v = whole(4) ? 4 : whole(2) ? 2 : 1, columns = 32 * v * LOOKUP_PIECES;
    const dim3 blocks((unsigned)((a.rows + 7) / 8), (a.dim + columns - 1) / columns);
    launch_pdl(v == 4 ? lookup_rows_kernel<S, T, 4> : v == 2 ? lookup_rows_kernel<S, T, 2> : lookup_rows_kernel<S, T, 1>, blocks, 256, 0, st, t, ids, o, a);
}

// ------------------------------------------------------------------------------------------------ sort
struct __align__(8) Pair {
    unsigned key, pos;        // id (vocab: outside the table), row
};

constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32;
constexpr int CHUNK_CTAS = 8, CHUNK_ROUNDS = 16, FEW_ROUNDS = 4;                              // CTAs of a cluster; pairs of a thread
constexpr unsigned CHUNK = SORT_THREADS * CHUNK_CTAS * CHUNK_ROUNDS;          // tokens of a cluster
constexpr int MAX_CHUNKS = 16;                                                // sorted lists that are merged
constexpr int DIGIT = 9, BINS = 1 << DIGIT;

struct SortArgs {
    const int32_t* ids;
    Pair* out;                // sorted lists, CHUNK apart
    unsigned n, vocab;
    int bits, sort_ctas;      // CTAs that sort; the others write zeros
    unsigned pos0;
    float* zero;
    size_t n_zero;
};

// zeros to p[0 .. n), by `parts` blocks of which this is number `part`
__device__ __forceinline__ void write_zeros(float* p, size_t n, size_t part, size_t parts) {
    const size_t head = min(n, (size_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / 4), vecs = (n - head) / 4;
    float4* v = reinterpret_cast<float4*>(p + head);
    for (size_t i = part * SORT_THREADS + threadIdx.x; i < vecs; i += parts * SORT_THREADS) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (part == 0 && threadIdx.x < 8) {
        const size_t tail0 = head + vecs * 4;
        if (threadIdx.x < head) p[threadIdx.x] = 0.f;
        if (threadIdx.x >= 4 && tail0 + threadIdx.x - 4 < n) p[tail0 + threadIdx.x - 4] = 0.f;
    }
}

template <int ROUNDS> struct SortShared {
    Pair items[SORT_THREADS * ROUNDS];
    unsigned short cnt[SORT_WARPS][BINS];      // a warp's pairs of a digit, then those of the warps before it
    unsigned tot[BINS];                        // the CTA's; read by the cluster
    unsigned first[BINS];                      // where the CTA's pairs of a digit start in the cluster's list
    unsigned wsum[SORT_WARPS];
};

// One radix sort a cluster.  A warp owns 32 * ROUNDS consecutive pairs and takes them 32 at a time: lanes of equal digits find each other by ballots,
// their rank is their place among them behind what the warp has counted of the digit.  All pairs are in registers when they are scattered, so
// one buffer suffices.
template <int ROUNDS> __global__ void __launch_bounds__(SORT_THREADS) sort_kernel(const SortArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    SortShared<ROUNDS>& s = *reinterpret_cast<SortShared<ROUNDS>*>(smem);
    pdl_wait();
    pdl_launch();
    if ((int)blockIdx.x >= a.sort_ctas) {
        write_zeros(a.zero, a.n_zero, blockIdx.x - a.sort_ctas, gridDim.x - a.sort_ctas);
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned rank = cluster.block_rank(), ctas = cluster.num_blocks(), chunk = blockIdx.x / ctas;
    const unsigned start = chunk * CHUNK, n = min(a.n - start, CHUNK);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned at0 = rank * (SORT_THREADS * ROUNDS) + warp * (32 * ROUNDS) + lane;       // place of round 0 in the cluster's list
    Pair p[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const unsigned i = at0 + k * 32;
        const unsigned id = i < n ? (unsigned)a.ids[start + i] : 0u;
        // what is not there sorts behind everything else
        p[k] = Pair{i >= n ? ~0u : id < a.vocab ? id : a.vocab, a.pos0 + start + i};
    }
    const int passes = (a.bits + DIGIT - 1) / DIGIT, step = (a.bits + passes - 1) / passes, bins = 1 << step;
    for (int pass = 0; pass < passes; ++pass) {
        const int sh = pass * step;
        for (int i = lane; i < bins / 2; i += 32) reinterpret_cast<unsigned*>(s.cnt[warp])[i] = 0;
        __syncwarp();
        unsigned place[ROUNDS];
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            const unsigned d = (p[k].key >> sh) & (bins - 1);
            unsigned same = 0xffffffffu;
            for (int b = 0; b < step; ++b) {
                const unsigned bit = (d >> b) & 1, vote = __ballot_sync(0xffffffffu, bit);
                same &= bit ? vote : ~vote;
            }
            const unsigned before = __popc(same & ((1u << lane) - 1u));
            const unsigned base = s.cnt[warp][d];
            __syncwarp();
            if (before == 0) s.cnt[warp][d] = (unsigned short)(base + __popc(same));
            __syncwarp();
            place[k] = base + before;
        }
        __syncthreads();
        if (tid < bins / 2 || tid == 0) {      // two digits a thread, packed: a CTA's count is at most 2^13
            unsigned* w = reinterpret_cast<unsigned*>(&s.cnt[0][0]) + tid;
            unsigned sum = 0, c[SORT_WARPS];
#pragma unroll
            for (int k = 0; k < SORT_WARPS; ++k) c[k] = w[k * (BINS / 2)];
#pragma unroll
            for (int k = 0; k < SORT_WARPS; ++k) {
                w[k * (BINS / 2)] = sum;
                sum += c[k];
            }
            s.tot[2 * tid] = sum & 0xffffu;
            s.tot[2 * tid + 1] = sum >> 16;
        }
        cluster.sync();
        unsigned all = 0, mine = 0;
        if (tid < bins) {
            unsigned t[CHUNK_CTAS];
#pragma unroll
            for (unsigned c = 0; c < CHUNK_CTAS; ++c) t[c] = c < ctas ? cluster.map_shared_rank(s.tot, c)[tid] : 0u;
#pragma unroll
            for (unsigned c = 0; c < CHUNK_CTAS; ++c) {
                mine += c < rank ? t[c] : 0u;
                all += t[c];
            }
        }
        unsigned incl = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        if (lane == 31) s.wsum[warp] = incl;
        __syncthreads();
        if (tid < bins) {
            unsigned b = 0;
            for (int k = 0; k < warp; ++k) b += s.wsum[k];
            s.first[tid] = b + incl - all + mine;
        }
        __syncthreads();
        const bool last = pass + 1 == passes;
        if (last) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // has read the other CTAs' totals
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            const unsigned d = (p[k].key >> sh) & (bins - 1);
            const unsigned g = s.first[d] + s.cnt[warp][d] + place[k];
            if (last) {
                if (g < n) a.out[start + g] = p[k];
            } else {
                cluster.map_shared_rank(s.items, g / (SORT_THREADS * ROUNDS))[g % (SORT_THREADS * ROUNDS)] = p[k];
            }
        }
        if (last) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // ... and they this one's, which may end now
        else cluster.sync();
        if (!last) {
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) p[k] = s.items[warp * (32 * ROUNDS) + k * 32 + lane];
        }
    }
}

// Sorted lists of CHUNK pairs (the last one shorter) into one.  Equal ids keep the order of the lists.  A pair's place is its own in its list and those of the
// largest prefixes of the others that go in front of it.  All searches take their steps together; the upper ones look at every SAMPLE-th key, which a block
// keeps in shared memory.
constexpr int SAMPLE = 512, SAMPLES = CHUNK / SAMPLE;

template <int LISTS> __global__ void __launch_bounds__(256) merge_kernel(const Pair* __restrict__ in, Pair* __restrict__ out, unsigned n) {
    __shared__ unsigned sample[LISTS * SAMPLES];
    pdl_wait();
    pdl_launch();
    for (unsigned i = threadIdx.x; i < LISTS * SAMPLES; i += 256) {
        const unsigned at = i * SAMPLE + SAMPLE - 1;         // the last key of a stretch
        sample[i] = at < n ? in[at].key : ~0u;
    }
    __syncthreads();
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const Pair p = in[i];
    const unsigned list = i / CHUNK;
    unsigned lo[LISTS];
    auto goes_before = [&](unsigned k, unsigned l) { return k < p.key || (k == p.key && l < list); };
#pragma unroll
    for (int l = 0; l < LISTS; ++l) lo[l] = 0;
#pragma unroll
    for (unsigned w = SAMPLES / 2; w; w >>= 1)
#pragma unroll
        for (int l = 0; l < LISTS; ++l)
            if (goes_before(sample[l * SAMPLES + lo[l] + w - 1], l)) lo[l] += w;
#pragma unroll
    for (int l = 0; l < LISTS; ++l)                          // the search so far ends one stretch short of a whole list
        if (goes_before(sample[l * SAMPLES + lo[l]], l)) ++lo[l];
#pragma unroll
    for (int l = 0; l < LISTS; ++l) lo[l] *= SAMPLE;
#pragma unroll
    for (unsigned w = SAMPLE / 2; w; w >>= 1) {
        unsigned k[LISTS];
#pragma unroll
        for (int l = 0; l < LISTS; ++l) {
            const unsigned at = l * CHUNK + lo[l] + w - 1;
            k[l] = lo[l] + w <= CHUNK && at < n ? in[at].key : ~0u;
        }
#pragma unroll
        for (int l = 0; l < LISTS; ++l)
            if (goes_before(k[l], l)) lo[l] += w;
    }
    unsigned at = i - list * CHUNK;
#pragma unroll
    for (int l = 0; l < LISTS; ++l)
        if ((unsigned)l != list) at += lo[l];
    out[at] = p;
}

// ------------------------------------------------------------------------------------------------ runs of equal ids
constexpr int RUN_WARPS = 8, COLS = 256, LANE_COLS = 8;

struct RunArgs {
    const Pair* s;
    const void* dy;
    size_t lddy;
    float *grad, *part;       // part [blocks][2][dim]: the run that came in over the block's start, the one that goes out over its end
    unsigned n, vocab;
    int dim, per_warp;        // sorted tokens of a warp, at most 32
    float scale;
    int add;
};

// column j of a lane: vectors of 8, or every 32nd
template <bool VEC> __device__ __forceinline__ int lane_col(int lane, int j) { return VEC ? lane * LANE_COLS + j : lane + 32 * j; }

template <typename T, bool VEC> struct Row {
    Vec<T> v[LANE_COLS / Vec<T>::N];
    T e[VEC ? 1 : LANE_COLS];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
        if (VEC) {
            if (lane * LANE_COLS < left)
#pragma unroll
                for (int i = 0; i < LANE_COLS / Vec<T>::N; ++i) {
                    if (i == 0 || lane * LANE_COLS + i * Vec<T>::N < left) v[i].load(p + lane * LANE_COLS, i);
                    else v[i].raw = decltype(v[i].raw){};
                }
        } else {
#pragma unroll
            for (int j = 0; j < LANE_COLS; ++j)
                if (lane + 32 * j < left) e[VEC ? 0 : j] = p[lane + 32 * j];
                else e[VEC ? 0 : j] = from_f<T>(0.f);
        }
    }
    __device__ __forceinline__ void get(float* f) const {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < LANE_COLS / Vec<T>::N; ++i) v[i].unpack(f + i * Vec<T>::N);
        } else {
#pragma unroll
            for (int j = 0; j < LANE_COLS; ++j) f[j] = to_f<T>(e[VEC ? 0 : j]);
        }
    }
};

// A row's sum into the gradient.  A call adds to every element at most once, so an addition at the memory gives the same bits in any order, and nobody waits
// for the old value.  (It takes numbers below 2^-126 for zero.)
__device__ __forceinline__ void put1(const RunArgs& a, float* g, float sum) {
    if (a.add) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(g), "f"(a.scale * sum) : "memory");
    else *g = a.scale * sum;
}
template <bool VEC> __device__ __forceinline__ void put_grad(const RunArgs& a, unsigned key, int c0, int lane, const float* f) {
    float* g = a.grad + (size_t)key * a.dim + c0;
    const int left = a.dim - c0;
    if (VEC) {
#pragma unroll
        for (int i = 0; i < LANE_COLS; i += 4)
            if (lane * LANE_COLS + i < left) {
                float* q = g + lane * LANE_COLS + i;
                if (a.add)
                    asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(q), "f"(a.scale * f[i]), "f"(a.scale * f[i + 1]),
                                 "f"(a.scale * f[i + 2]), "f"(a.scale * f[i + 3])
                                 : "memory");
                else *reinterpret_cast<float4*>(q) = make_float4(a.scale * f[i], a.scale * f[i + 1], a.scale * f[i + 2], a.scale * f[i + 3]);
            }
    } else {
#pragma unroll
        for (int j = 0; j < LANE_COLS; ++j)
            if (lane + 32 * j < left) put1(a, g + lane + 32 * j, f[j]);
    }
}

constexpr unsigned NO_KEY = ~0u;

template <typename T, bool VEC> __global__ void __launch_bounds__(RUN_WARPS * 32, VEC && sizeof(T) == 2 ? 4 : 2) runs_kernel(const RunArgs a) {
    // of every warp the sum that came in over its start and the one that goes out over its end
    __shared__ float open[RUN_WARPS][2][COLS];
    __shared__ unsigned first_key[RUN_WARPS], last_key[RUN_WARPS];
    constexpr int AHEAD = 8;
    pdl_wait();
    pdl_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c0 = blockIdx.x * COLS, left = a.dim - c0;
    const unsigned block0 = blockIdx.y * (RUN_WARPS * a.per_warp), w0 = block0 + warp * a.per_warp;
    const unsigned w1 = min(w0 + a.per_warp, a.n);
    const unsigned i = w0 + lane, i_behind = w0 + a.per_warp;
    // all requested at once: the warp's tokens and the keys around them
    Pair p{NO_KEY, 0};
    if (i < w1) p = a.s[i];
    unsigned before = w0 && w0 < a.n ? a.s[w0 - 1].key : NO_KEY, behind = i_behind < a.n ? a.s[i_behind].key : NO_KEY;
    if (p.key >= a.vocab) p.key = NO_KEY;                       // tokens outside the table are no run
    if (before >= a.vocab) before = NO_KEY;
    if (behind >= a.vocab) behind = NO_KEY;
    const int count = __popc(__ballot_sync(0xffffffffu, p.key != NO_KEY));       // tokens outside the table are last
    const unsigned k_first = __shfl_sync(0xffffffffu, p.key, 0), k_last = __shfl_sync(0xffffffffu, p.key, max(count - 1, 0));
    const bool came = count && before == k_first, goes = count && behind == k_last;
    if (lane == 0) {
        first_key[warp] = came ? k_first : NO_KEY;
        last_key[warp] = goes ? k_last : NO_KEY;
    }
    float acc[LANE_COLS];
    unsigned key = k_first;
    bool at_start = true;                            // the run at hand is the warp's first
#pragma unroll
    for (int j = 0; j < LANE_COLS; ++j) acc[j] = 0.f;
    auto done = [&](bool at_end) {
        if (at_start && came) {
#pragma unroll
            for (int j = 0; j < LANE_COLS; ++j) open[warp][0][lane_col<VEC>(lane, j)] = acc[j];
        } else if (at_end && goes) {
#pragma unroll
            for (int j = 0; j < LANE_COLS; ++j) open[warp][1][lane_col<VEC>(lane, j)] = acc[j];
        } else {
            put_grad<VEC>(a, key, c0, lane, acc);
        }
    };
    for (int e0 = 0; e0 < count; e0 += AHEAD) {
        Row<T, VEC> row[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const unsigned pos = __shfl_sync(0xffffffffu, p.pos, (e0 + e) & 31);
            if (e0 + e < count) row[e].load(static_cast<const T*>(a.dy) + (size_t)pos * a.lddy + c0, lane, left);
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const unsigned k = __shfl_sync(0xffffffffu, p.key, (e0 + e) & 31);
            if (e0 + e >= count) continue;
            float f[LANE_COLS];
            row[e].get(f);
            if (k != key) {
                done(false);
                key = k;
                at_start = false;
#pragma unroll
                for (int j = 0; j < LANE_COLS; ++j) acc[j] = f[j];
            } else {
#pragma unroll
                for (int j = 0; j < LANE_COLS; ++j) acc[j] += f[j];
            }
        }
    }
    if (count) done(true);
    __syncthreads();
    // One thread a column joins the warps' open ends in order.  A run that only came in and goes out again has its sum in the first place.
    const int c = threadIdx.x;
    if (c >= left) return;
    float* part = a.part + (size_t)blockIdx.y * 2 * a.dim + c0 + c;
    float sum = 0.f;
    bool held = false, from_before = false;          // a run is open; it began in front of the block
    for (int w = 0; w < RUN_WARPS; ++w) {
        const unsigned kf = first_key[w], kl = last_key[w];
        if (kf != NO_KEY) {
            if (!held) from_before = true;           // w == 0
            sum += open[w][0][c];
            held = true;
            const bool through = kl == kf;           // sorted: the warp holds nothing else
            if (!through) {
                if (from_before) part[0] = sum;
                else put1(a, a.grad + (size_t)kf * a.dim + c0 + c, sum);
                held = false;
                from_before = false;
                sum = 0.f;
            }
            if (through) continue;
        }
        if (kl != NO_KEY) {
            sum = open[w][1][c];
            held = true;
            from_before = false;
        }
    }
    if (held) part[from_before ? 0 : a.dim] = sum;
}

// The run that goes out over the end of block b, if it began there: its parts in order.  The keys it takes to know that are requested together: those around the
// block, and the first ones of the 32 blocks behind.
template <bool VEC> __global__ void __launch_bounds__(256) join_kernel(const RunArgs a, unsigned blocks) {
    pdl_wait();
    pdl_launch();
    const unsigned b = blockIdx.y * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, c0 = blockIdx.x * COLS, left = a.dim - c0;
    const unsigned per = RUN_WARPS * a.per_warp;
    if (b + 1 >= blocks) return;
    const unsigned key = a.s[(b + 1) * per - 1].key, first = a.s[b * per].key, before = b ? a.s[b * per - 1].key : NO_KEY;
    unsigned next = b + 1 + lane < blocks ? a.s[(b + 1 + lane) * per].key : NO_KEY;
    if (key >= a.vocab || (first == key && before == key) || __shfl_sync(0xffffffffu, next, 0) != key) return;
    Row<float, VEC> r;
    float acc[LANE_COLS], f[LANE_COLS];
    r.load(a.part + ((size_t)b * 2 + 1) * a.dim + c0, lane, left);
    r.get(acc);
    for (unsigned t = b + 1;;) {
        const unsigned m = __ballot_sync(0xffffffffu, next == key);
        const int k = m == 0xffffffffu ? 32 : __ffs(~m) - 1;
        constexpr int AHEAD = 8;
        for (int e0 = 0; e0 < k; e0 += AHEAD) {
            Row<float, VEC> q[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e)
                if (e0 + e < k) q[e].load(a.part + (size_t)(t + e0 + e) * 2 * a.dim + c0, lane, left);
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                if (e0 + e >= k) continue;
                q[e].get(f);
#pragma unroll
                for (int j = 0; j < LANE_COLS; ++j) acc[j] += f[j];
            }
        }
        t += 32;
        if (k < 32 || t >= blocks) break;
        next = t + lane < blocks ? a.s[(t + lane) * per].key : NO_KEY;
    }
    put_grad<VEC>(a, key, c0, lane, acc);
}

int bits_of(unsigned v) {
    int b = 0;
    while (v >> b) ++b;
    return b;
}

// Sorted tokens of a warp: as many as leave some 4 warps for each of the 4 schedulers of 148 multiprocessors, at most 32.  Fewer make more open ends, more make
// longer chains of requests.
constexpr size_t FEW_WARPS = 2368;
int per_warp_of(size_t rows, int dim) {
    const size_t slabs = ((size_t)dim + COLS - 1) / COLS;
    int r = 32;
    while (r > 4 && (rows + r - 1) / r * slabs < FEW_WARPS) r >>= 1;
    return r;
}
size_t run_blocks(size_t rows, int per_warp) { return (rows + RUN_WARPS * per_warp - 1) / (RUN_WARPS * per_warp); }
// The most blocks that `rows` rows or fewer take.  From some row count on warps have twice as many tokens and there are half as many blocks: those of
// each length are largest at the last row count that has it.
size_t most_blocks(size_t rows, int dim) {
    const size_t slabs = ((size_t)dim + COLS - 1) / COLS;
    size_t most = run_blocks(rows, per_warp_of(rows, dim));
    for (int r = 4; r < 32; r <<= 1) most = std::max(most, run_blocks(std::min(rows, 2 * r * ((FEW_WARPS - 1) / slabs)), r));
    return most;
}

constexpr size_t MAX_ROWS = ((size_t)1 << 31) - 1, MAX_ELEMS = (size_t)1 << 40;
constexpr int MAX_DIM = 1 << 20;

int bad_shape(const void* ids, size_t rows, int vocab, int dim, const void* p, size_t ld, int dtype) {
    if ((!ids || !p) && rows) return report_error(AST_ERR_ARG, "null argument");
    if (dtype != AST_F32 && dtype != AST_BF16) return report_error(AST_ERR_ARG, "bad dtype");
    if (rows > MAX_ROWS || vocab < 1 || dim < 1 || dim > MAX_DIM || (size_t)vocab > MAX_ELEMS / dim || (rows && (size_t)dim > MAX_ELEMS / rows))
        return report_error(AST_ERR_ARG, "rows, vocab or dim out of range");
    if (ld < (size_t)dim || (rows && ld > MAX_ELEMS / rows)) return report_error(AST_ERR_ARG, "the row stride is out of range");
    if (reinterpret_cast<uintptr_t>(p) % (dtype == AST_F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(ids) % 4)
        return report_error(AST_ERR_ARG, "a tensor does not start at an element of its type");
    return AST_OK;
}
int launched() {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AST_OK : report_error(AST_ERR_CUDA, cudaGetErrorString(e));
}

// What a gradient of so many tokens needs: at most `part` tokens are sorted at a time, by pairs (two lists where they are merged), then the partial
// rows of the blocks' ends.  `bytes` suffices for every smaller number of tokens as well.
struct BackwardPlan {
    size_t part, pair_bytes, bytes;
    int per_warp;
    BackwardPlan(size_t rows, int dim) {
        part = std::min(rows, (size_t)MAX_CHUNKS * CHUNK);
        part += part & 1;                                  // the second list and the partial rows start at 16 bytes
        per_warp = per_warp_of(part, dim);
        pair_bytes = part * sizeof(Pair) * (part > CHUNK ? 2 : 1);
        bytes = rows ? pair_bytes + most_blocks(part, dim) * 2 * dim * sizeof(float) : 0;
    }
};

// One launch: clusters that sort, CHUNK tokens each, and blocks that write zeros.  A single list takes as many CTAs as leave four pairs a thread, 8 at most.
void sort_tokens(const SortArgs& s0, cudaStream_t st) {
    SortArgs s = s0;
    const bool few = s.n <= SORT_THREADS * FEW_ROUNDS * CHUNK_CTAS;
    int ctas = 1;
    while (ctas < CHUNK_CTAS && (size_t)ctas * SORT_THREADS * FEW_ROUNDS < s.n) ctas *= 2;
    const int chunks = (int)((s.n + CHUNK - 1) / CHUNK);
    s.sort_ctas = ctas * chunks;
    // blocks for the zeros, of 256 KB: many, so that the multiprocessors that have sorted take their share
    int zero = (int)std::min<size_t>(32768, (s.n_zero + 65535) / 65536);
    zero = (zero + ctas - 1) / ctas * ctas;
    LaunchScope ls(K_EMBED_SORT, 12.0 * s.n + 4.0 * s.n_zero, 0.0, st);
    if (few) {
        smem_limit_once<140>(sort_kernel<FEW_ROUNDS>, (int)sizeof(SortShared<FEW_ROUNDS>));
        launch_pdl_cluster(sort_kernel<FEW_ROUNDS>, s.sort_ctas + zero, SORT_THREADS, ctas, sizeof(SortShared<FEW_ROUNDS>), st, s);
    } else {
        smem_limit_once<141>(sort_kernel<CHUNK_ROUNDS>, (int)sizeof(SortShared<CHUNK_ROUNDS>));
        launch_pdl_cluster(sort_kernel<CHUNK_ROUNDS>, s.sort_ctas + zero, SORT_THREADS, ctas, sizeof(SortShared<CHUNK_ROUNDS>), st, s);
    }
}

}  // namespace
}  // namespace ast

using namespace ast;

extern "C" {

int asteroid_embedding_forward(const void* table, int table_dtype, const int32_t* ids, size_t rows, int vocab, int dim, float scale, void* y, size_t ldy, int dtype,
                               void* stream) {
    int rc = bad_shape(ids, rows, vocab, dim, y, ldy, dtype);
    if (rc) return rc;
    if (!table) return report_error(AST_ERR_ARG, "null argument");
    if (table_dtype != AST_F32 && table_dtype != AST_BF16) return report_error(AST_ERR_ARG, "bad table dtype");
    if (reinterpret_cast<uintptr_t>(table) % (table_dtype == AST_F32 ? 4 : 2)) return report_error(AST_ERR_ARG, "a tensor does not start at an element of its type");
    if (!rows) return AST_OK;
    typedef __nv_bfloat16 bf;
    cudaStream_t st = (cudaStream_t)stream;
    const bool tf = table_dtype == AST_F32, yf = dtype == AST_F32;
    LookupShape a{};
    a.rows = rows; a.ldy = ldy; a.vocab = vocab; a.dim = dim; a.scale = scale;
    LaunchScope ls(K_EMBED_FWD, rows * (4.0 + dim * ((tf ? 4.0 : 2.0) + (yf ? 4.0 : 2.0))), 0.0, st);
    if (tf && yf) launch_lookup<float, float>(table, ids, y, a, st);
    else if (tf) launch_lookup<float, bf>(table, ids, y, a, st);
    else if (yf) launch_lookup<bf, float>(table, ids, y, a, st);
    else launch_lookup<bf, bf>(table, ids, y, a, st);
    return launched();
}

size_t asteroid_embedding_workspace(size_t rows, int dim) {
    if (rows > MAX_ROWS || dim < 1 || dim > MAX_DIM || rows * dim > MAX_ELEMS) return 0;
    return BackwardPlan(rows, dim).bytes;
}

int asteroid_embedding_backward(const int32_t* ids, const void* dy, size_t lddy, size_t rows, int vocab, int dim, float scale, int dtype, float* grad, int accumulate,
                                void* workspace, size_t workspace_bytes, void* stream) {
    int rc = bad_shape(ids, rows, vocab, dim, dy, lddy, dtype);
    if (rc) return rc;
    if (!grad) return report_error(AST_ERR_ARG, "null argument");
    if (reinterpret_cast<uintptr_t>(grad) % 4) return report_error(AST_ERR_ARG, "a tensor does not start at an element of its type");
    const BackwardPlan plan(rows, dim);
    if (plan.bytes && (!workspace || workspace_bytes < plan.bytes)) return report_error(AST_ERR_ARG, "the workspace is too small");
    if (plan.bytes && reinterpret_cast<uintptr_t>(workspace) % 16) return report_error(AST_ERR_ARG, "a workspace must start at a 16-byte boundary");
    cudaStream_t st = (cudaStream_t)stream;
    const double esz = dtype == AST_F32 ? 4.0 : 2.0;
    bool zero = !accumulate, add = accumulate != 0;
    // at most `plan.part` tokens at a time; the gradients of further ones are added
    for (size_t r0 = 0; r0 < rows || zero; r0 += plan.part) {
        const unsigned n = (unsigned)std::min(plan.part, rows - r0);
        Pair* sorted = static_cast<Pair*>(workspace);
        {
            SortArgs s{};
            s.ids = ids ? ids + r0 : nullptr; s.out = sorted; s.n = n; s.vocab = (unsigned)vocab; s.bits = bits_of((unsigned)vocab); s.pos0 = (unsigned)r0;
            s.zero = grad; s.n_zero = zero ? (size_t)vocab * dim : 0;
            sort_tokens(s, st);
        }
        zero = false;
        if (!n) break;
        if (n > CHUNK) {
            LaunchScope ls(K_EMBED_SORT, 16.0 * n, 0.0, st);
            const unsigned lists = (n + CHUNK - 1) / CHUNK;
            launch_pdl(lists <= 2 ? merge_kernel<2> : lists <= 4 ? merge_kernel<4> : lists <= 8 ? merge_kernel<8> : merge_kernel<MAX_CHUNKS>, (n + 255) / 256, 256, 0, st,
                       sorted, sorted + plan.part, n);
            sorted += plan.part;
        }
        RunArgs a{};
        a.s = sorted; a.dy = dy; a.lddy = lddy; a.grad = grad; a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.pair_bytes);
        a.n = n; a.vocab = (unsigned)vocab; a.dim = dim; a.per_warp = plan.per_warp; a.scale = scale; a.add = add;
        const unsigned blocks = (unsigned)run_blocks(n, a.per_warp), slabs = (unsigned)((dim + COLS - 1) / COLS);
        const int N = dtype == AST_F32 ? 4 : 8;
        const bool vec = dim % N == 0 && lddy % N == 0 && (reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(grad)) % 16 == 0;
        {
            LaunchScope ls(K_EMBED_BWD, n * (8.0 + dim * esz), (double)n * dim, st);
            const dim3 grid(slabs, blocks);              // the columns of the same rows at the same time
            if (dtype == AST_F32) launch_pdl(vec ? runs_kernel<float, true> : runs_kernel<float, false>, grid, RUN_WARPS * 32, 0, st, a);
            else launch_pdl(vec ? runs_kernel<__nv_bfloat16, true> : runs_kernel<__nv_bfloat16, false>, grid, RUN_WARPS * 32, 0, st, a);
        }
        if (blocks > 1) {
            LaunchScope ls(K_EMBED_BWD, 0.0, 0.0, st);
            launch_pdl(vec ? join_kernel<true> : join_kernel<false>, dim3(slabs, (blocks + 7) / 8), 256, 0, st, a, blocks);
        }
        add = true;
    }
    return launched();
}

}  // extern "C"
