// Activations packed into 8-bit checkpoints, read back, and used by an activation layer's backward (the form: ckpt8.cuh).
//
// All passes are elementwise over groups of 32 columns and bound by memory: a thread owns one 16-byte vector of the storage type (4 or 8
// values), the 8 or 4 lanes of a group find its largest magnitude by shuffles, and every tensor is read and written once.  Instructions are next: a SiLU step
// of 16 384 x 2048 bfloat16 numbers takes 56 us, 84 % of the memory's rate, with the schedulers busy in two cycles of three; packing and unpacking 100 352 x 256 26 us, of
// which memory needs 20.
#include "../../include/asteroid.h"
#include "ckpt8.cuh"
#include "kernels.h"

namespace ast {
namespace {

using namespace q8;

// Dense rows of whole groups; rows of whole vectors; rows of whole pieces of 8 or 4 bytes; anything else.  (300 000 rows of 100 bfloat16 numbers: 148 us by single
// values a lane, 64 by pieces of 8 bytes.)
enum { FLAT = 0, ROWS = 1, PIECE8 = 2, PIECE4 = 3, SINGLE = 4 };
constexpr int THREADS = 256, PER_THREAD = 2, BLOCK = THREADS * PER_THREAD;

struct Args {
    const void *x, *dy;
    void *out, *codes, *exps;
    size_t ldx, lddy, ldo;
    size_t vecs, rows;        // vecs = rows * vecs_per_row
    unsigned vecs_per_row;    // vectors of a row of whole groups
    unsigned cols;
    // a block has up to BLOCK vectors: rows_per_block whole rows, or one of the col_blocks stretches of a row; inv: 2^20 / vectors of its row, rounded up
    unsigned rows_per_block, col_blocks, inv;
};

// value and slope of the activations; float32 storage takes the functions to float32 accuracy, bfloat16 storage to well below its rounding
// (2^x and the reciprocal to 2 and 1 units, their results below 2^-126 zero: the forms that keep them take twice the instructions, which is what bounds these passes).
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + exp(-x)), and what it is short of 1.  Far left of zero x * sigmoid(x) is a normal number where the sigmoid no longer is one: below -87.3 it is a multiple of 2^-149.  float32
// forms it from exp(-|x|), which underflows as it does instead of overflowing before; bfloat16 shifts the range of the exponential and the
// reciprocal, whose own numbers must be normal, by 2^32.  (16 384 x 2048, forward and backward: float32 101 and 104 us, bfloat16 54.6 and 54.9.)
template <typename T> struct Sigmoid {
    float s, rest;
    __device__ __forceinline__ explicit Sigmoid(float x) {
        const float e = expf(-fabsf(x)), q = 1.f / (1.f + e);
        s = x < 0.f ? e * q : q;
        rest = 1.f - s;
    }
};
template <> struct Sigmoid<__nv_bfloat16> {
    float s, rest;
    __device__ __forceinline__ explicit Sigmoid(float x) {
        const float r = fast_rcp(fast_exp2(fmaf(x, -1.44269504f, -32.f)) + 0x1p-32f);
        s = r * 0x1p-32f;
        rest = fmaf(r, -0x1p-32f, 1.f);
    }
};

// The normal distribution function at x, and exp(-x^2 / 2)
struct Normal {
    float cdf, bell;
};
template <typename T> __device__ __forceinline__ Normal normal(float x) { return Normal{0.5f * erfcf(-0.70710678118654752f * x), expf(-0.5f * x * x)}; }
// For bfloat16 storage, from the bell: the smaller tail is bell * erfcx(z) / 2, z = |x| / sqrt 2, and erfcx(z) = exp(z^2) erfc(z) is fitted by t P(t), t = 1 / (1 +
// 0.55 z), to 4.3e-6 of itself for all z >= 0 (least squares with weights that even out the relative error).  With erfcf the pass was bound by its instructions:
// 134 us for a step of 30000 x 1024, 66 so.
template <> __device__ __forceinline__ Normal normal<__nv_bfloat16>(float x) {
    const float bell = fast_exp2(-0.72134752f * x * x), t = fast_rcp(fmaf(0.38890873f, fabsf(x), 1.f));
    float p = 0.0494244285f;
    p = fmaf(p, t, -0.1509267688f);
    p = fmaf(p, t, 0.0885909051f);
    p = fmaf(p, t, 0.0693081692f);
    p = fmaf(p, t, 0.1333594620f);
    p = fmaf(p, t, 0.1550938487f);
    p = fmaf(p, t, 0.1551520824f);
    const float tail = bell * t * p;
    return Normal{x < 0.f ? tail : 1.f - tail, bell};
}

template <typename T, int ACT> __device__ __forceinline__ float value(float x) {
    if (ACT == AST_RELU) return x < 0.f ? 0.f : x;
    if (ACT == AST_RELU6) return x < 0.f ? 0.f : x > 6.f ? 6.f : x;
    if (ACT == AST_SILU) {
        const Sigmoid<T> g(x);
        return x * g.s;
    }
    if (ACT == AST_GELU) return x * normal<T>(x).cdf;
    return x;
}
// dy * act'(x); a gradient that the activation does not pass on is zero whatever it is, one of an x that reads as NaN is NaN
template <typename T, int ACT> __device__ __forceinline__ float slope(float x, float dy) {
    if (ACT == AST_RELU) return x > 0.f ? dy : x == x ? 0.f : x;
    if (ACT == AST_RELU6) return x > 0.f && x < 6.f ? dy : x == x ? 0.f : x;
    if (ACT == AST_SILU) {
        const Sigmoid<T> g(x);
        return dy * (g.s * fmaf(x, g.rest, 1.f));
    }
    const Normal n = normal<T>(x);
    return dy * fmaf(0.3989422804014327f * x, n.bell, n.cdf);
}

template <int MODE> struct Piece {
    typedef uint2 type;
};
template <> struct Piece<PIECE4> {
    typedef unsigned type;
};
// Rows of bfloat16 numbers that start anywhere: a warp's 32 vectors are taken value by value, 32 consecutive ones of the (mostly one) row at a time, and change hands in shared memory, 16
// bytes a lane.  (30 000 rows of 999 bfloat16 numbers, packed and unpacked: 112 us with each lane fetching its own 8, 68 so; four float32
// numbers a lane are faster by themselves, 68 and 76.)  Whole warps call it.
template <typename T> struct Singles {
    static constexpr int N = Vec<T>::N, VECS = 32 / N;
    size_t base;              // of this lane's vector
    unsigned count;           // its values inside the tensor
    __device__ __forceinline__ Singles(size_t ld, size_t row, unsigned c, unsigned cols, bool in) : base(in ? row * ld + c : 0), count(in ? min(cols - c, (unsigned)N) : 0u) {}
    // value i * 32 + lane of the warp's: its place, or none
    __device__ __forceinline__ bool at(int i, size_t* place) const {
        const int lane = threadIdx.x & 31, from = i * VECS + lane / N;
        const unsigned n = __shfl_sync(0xffffffffu, count, from);
        *place = __shfl_sync(0xffffffffu, (unsigned long long)base, from) + lane % N;
        return (unsigned)(lane % N) < n;
    }
    __device__ __forceinline__ void load(const T* p, T* hand, float* f) const {
        const int lane = threadIdx.x & 31;
        T v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            size_t place;
            v[i] = T{};
            if (at(i, &place)) v[i] = p[place];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) hand[i * 32 + lane] = v[i];
        __syncwarp();
        Vec<T> r;
        r.load(hand, lane);
        r.unpack(f);
    }
    __device__ __forceinline__ void store(T* p, T* hand, const float* f) const {
        const int lane = threadIdx.x & 31;
        Vec<T> r;
        r.pack(f);
        __syncwarp();
        r.store(hand, lane);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            size_t place;
            if (at(i, &place)) p[place] = hand[i * 32 + lane];
        }
    }
};
template <typename T, int MODE>
__device__ __forceinline__ void load(const void* p, size_t ld, size_t row, unsigned c, unsigned cols, size_t v, bool in, T* hand, float* f) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = 0.f;
    if (MODE == SINGLE && sizeof(T) == 2) {
        Singles<T>(ld, row, c, cols, in).load(static_cast<const T*>(p), hand, f);
    } else if (MODE == SINGLE) {
        const T* q = static_cast<const T*>(p) + row * ld + c;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (in && c + i < cols) f[i] = to_f<T>(q[i]);
    } else if (MODE == PIECE8 || MODE == PIECE4) {
        typedef typename Piece<MODE>::type P;
        constexpr int E = sizeof(P) / sizeof(T);
        const P* q = reinterpret_cast<const P*>(static_cast<const T*>(p) + row * ld + c);
        Vec<T> r;
        r.raw = decltype(r.raw){};
        P* const d = reinterpret_cast<P*>(&r.raw);
#pragma unroll
        for (int i = 0; i < N / E; ++i)
            if (in && c + i * E < cols) d[i] = q[i];
        r.unpack(f);
    } else if (in) {
        Vec<T> r;
        r.load(static_cast<const T*>(p) + (MODE == FLAT ? v * N : row * ld + c), 0);
        r.unpack(f);
    }
}
template <typename T, int MODE>
__device__ __forceinline__ void store(void* p, size_t ld, size_t row, unsigned c, unsigned cols, size_t v, bool in, T* hand, const float* f) {
    constexpr int N = Vec<T>::N;
    if (MODE == SINGLE && sizeof(T) == 2) {
        Singles<T>(ld, row, c, cols, in).store(static_cast<T*>(p), hand, f);
    } else if (MODE == SINGLE) {
        T* q = static_cast<T*>(p) + row * ld + c;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (in && c + i < cols) q[i] = from_f<T>(f[i]);
    } else if (MODE == PIECE8 || MODE == PIECE4) {
        typedef typename Piece<MODE>::type P;
        constexpr int E = sizeof(P) / sizeof(T);
        P* q = reinterpret_cast<P*>(static_cast<T*>(p) + row * ld + c);
        Vec<T> r;
        r.pack(f);
        const P* const d = reinterpret_cast<const P*>(&r.raw);
#pragma unroll
        for (int i = 0; i < N / E; ++i)
            if (in && c + i * E < cols) q[i] = d[i];
    } else if (in) {
        Vec<T> r;
        r.pack(f);
        r.store(static_cast<T*>(p) + (MODE == FLAT ? v * N : row * ld + c), 0);
    }
}

// Bits of the largest magnitude.  bfloat16 values by pairs: the upper halves of two floats as one word.
template <typename T> __device__ __forceinline__ unsigned largest(const float* f) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    return top;
}
template <> __device__ __forceinline__ unsigned largest<__nv_bfloat16>(const float* f) {
    unsigned t = 0;
#pragma unroll
    for (int i = 0; i < 8; i += 2) t = __vmaxu2(t, __byte_perm(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), 0x7632) & 0x7fff7fffu);
    return max(t << 16, t & 0xffff0000u);
}

// The block's vector u: its index, row and first column, and whether there is one.  Groups start at multiples of their number of lanes.
template <typename T, int MODE> __device__ __forceinline__ bool place(const Args& a, unsigned u, size_t* v, size_t* row, unsigned* c) {
    if (MODE == FLAT) {
        *v = (size_t)blockIdx.x * BLOCK + u;
        *row = 0;
        *c = 0;
        return *v < a.vecs;
    }
    unsigned rb = blockIdx.x, c0 = 0;
    if (a.col_blocks > 1) {
        rb = blockIdx.x / a.col_blocks;
        c0 = (blockIdx.x - rb * a.col_blocks) * BLOCK;
    }
    const unsigned width = min(a.vecs_per_row - c0, (unsigned)BLOCK), r = (u * a.inv) >> 20;         // u, the row's vectors <= 512: exact; 0 where a row has more
    const unsigned cv = c0 + u - r * width;
    *row = (size_t)rb * a.rows_per_block + r;
    *v = *row * a.vecs_per_row + cv;
    *c = cv * Vec<T>::N;
    return u < a.rows_per_block * width && *row < a.rows;
}

template <typename T, int MODE, int ACT> __global__ void __launch_bounds__(THREADS) forward_kernel(const Args a) {
    constexpr int N = Vec<T>::N, LANES = GROUP / N;
    __shared__ __align__(16) T hands[MODE == SINGLE && sizeof(T) == 2 ? THREADS * N : 1];
    T* const hand = MODE == SINGLE && sizeof(T) == 2 ? hands + (threadIdx.x & ~31u) * N : nullptr;        // of this warp
    pdl_wait();
    pdl_launch();
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        size_t v, row;
        unsigned c;
        const bool live = place<T, MODE>(a, j * THREADS + threadIdx.x, &v, &row, &c), in = live && (MODE == FLAT || c < a.cols);
        float f[N];
        load<T, MODE>(a.x, a.ldx, row, c, a.cols, v, in, hand, f);
        unsigned top = largest<T>(f);
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const unsigned s = exp_byte(top);
        const float m = to_code(s);
        if (live) {
            unsigned w[N / 4];
            if (s < 254u) {
#pragma unroll
                for (int i = 0; i < N / 4; ++i) w[i] = pack4(code(f[4 * i], m), code(f[4 * i + 1], m), code(f[4 * i + 2], m), code(f[4 * i + 3], m));
            } else {
#pragma unroll
                for (int i = 0; i < N / 4; ++i)
                    w[i] = s == NOT_FINITE ? 0u : pack4(code_sat(f[4 * i], m), code_sat(f[4 * i + 1], m), code_sat(f[4 * i + 2], m), code_sat(f[4 * i + 3], m));
            }
            if (N == 4) static_cast<unsigned*>(a.codes)[v] = w[0];
            else static_cast<uint2*>(a.codes)[v] = make_uint2(w[0], w[N / 4 - 1]);
            if ((v & (LANES - 1)) == 0) static_cast<unsigned char*>(a.exps)[v / LANES] = (unsigned char)s;
        }
        if (ACT) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = value<T, ACT>(f[i]);
            store<T, MODE>(a.out, a.ldo, row, c, a.cols, v, in, hand, f);
        }
    }
}

template <typename T, int MODE, int ACT> __global__ void __launch_bounds__(THREADS) backward_kernel(const Args a) {
    constexpr int N = Vec<T>::N, LANES = GROUP / N;
    __shared__ __align__(16) T hands[MODE == SINGLE && sizeof(T) == 2 ? THREADS * N : 1];
    T* const hand = MODE == SINGLE && sizeof(T) == 2 ? hands + (threadIdx.x & ~31u) * N : nullptr;        // of this warp
    pdl_wait();
    pdl_launch();
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        size_t v, row;
        unsigned c;
        const bool in = place<T, MODE>(a, j * THREADS + threadIdx.x, &v, &row, &c) && (MODE == FLAT || c < a.cols);
        if (MODE != SINGLE && !in) continue;
        unsigned w[2] = {0u, 0u};
        if (!in) {
        } else if (N == 4) w[0] = static_cast<const unsigned*>(a.codes)[v];
        else {
            const uint2 t = static_cast<const uint2*>(a.codes)[v];
            w[0] = t.x;
            w[1] = t.y;
        }
        const float m = to_value(in ? static_cast<const unsigned char*>(a.exps)[v / LANES] : 8u);
        float f[N], g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = code_f(flip(w[i / 4]), i & 3) * m;
        if (ACT) {
            load<T, MODE>(a.dy, a.lddy, row, c, a.cols, v, in, hand, g);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = slope<T, ACT>(f[i], g[i]);
        }
        store<T, MODE>(a.out, a.ldo, row, c, a.cols, v, in, hand, f);
    }
}

template <typename T, int MODE> void launch_mode(bool fwd, int act, const Args& a, cudaStream_t st) {
    const unsigned blocks = MODE == FLAT ? (unsigned)((a.vecs + BLOCK - 1) / BLOCK) : (unsigned)((a.rows + a.rows_per_block - 1) / a.rows_per_block * a.col_blocks);
    auto go = [&](auto* k) { launch_pdl(k, blocks, THREADS, 0, st, a); };
    switch (act) {
        case AST_RELU: return fwd ? go(forward_kernel<T, MODE, AST_RELU>) : go(backward_kernel<T, MODE, AST_RELU>);
        case AST_RELU6: return fwd ? go(forward_kernel<T, MODE, AST_RELU6>) : go(backward_kernel<T, MODE, AST_RELU6>);
        case AST_SILU: return fwd ? go(forward_kernel<T, MODE, AST_SILU>) : go(backward_kernel<T, MODE, AST_SILU>);
        case AST_GELU: return fwd ? go(forward_kernel<T, MODE, AST_GELU>) : go(backward_kernel<T, MODE, AST_GELU>);
        default: return fwd ? go(forward_kernel<T, MODE, 0>) : go(backward_kernel<T, MODE, 0>);
    }
}

size_t groups_of(int cols) { return ((size_t)cols + GROUP - 1) / GROUP; }

template <typename T> void launch(bool fwd, int act, Args a, size_t rows, int cols, cudaStream_t st) {
    constexpr int N = Vec<T>::N;
    const size_t vpr = groups_of(cols) * (GROUP / N);
    a.vecs = rows * vpr;
    a.vecs_per_row = (unsigned)vpr;
    a.cols = (unsigned)cols;
    a.rows = rows;
    const unsigned width = (unsigned)(vpr < BLOCK ? vpr : BLOCK);
    a.rows_per_block = BLOCK / width;
    a.col_blocks = (unsigned)((vpr + BLOCK - 1) / BLOCK);
    a.inv = ((1u << 20) + width - 1) / width;
    // rows that start, and end, at multiples of `bytes`
    auto whole = [&](const void* p, size_t ld, size_t bytes) { return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * sizeof(T) % bytes == 0); };
    auto all = [&](size_t bytes) { return cols * sizeof(T) % bytes == 0 && whole(a.x, a.ldx, bytes) && whole(a.dy, a.lddy, bytes) && whole(a.out, a.ldo, bytes); };
    auto dense = [&](const void* p, size_t ld) { return !p || ld == (size_t)cols; };
    if (all(16) && cols % GROUP == 0 && dense(a.x, a.ldx) && dense(a.dy, a.lddy) && dense(a.out, a.ldo)) launch_mode<T, FLAT>(fwd, act, a, st);
    else if (all(16)) launch_mode<T, ROWS>(fwd, act, a, st);
    else if (all(8)) launch_mode<T, PIECE8>(fwd, act, a, st);
    else if (sizeof(T) == 2 && all(4)) launch_mode<T, sizeof(T) == 2 ? PIECE4 : SINGLE>(fwd, act, a, st);
    else launch_mode<T, SINGLE>(fwd, act, a, st);
}

}  // namespace

void ckpt8_forward(int dtype, int act, const void* x, size_t ldx, size_t rows, int cols, void* y, size_t ldy, void* codes, void* exps, cudaStream_t st) {
    if (!rows) return;
    Args a{};
    a.x = x; a.ldx = ldx; a.out = act ? y : nullptr; a.ldo = ldy; a.codes = codes; a.exps = exps;
    const double n = (double)rows * cols, e = dtype == AST_F32 ? 4 : 2;
    LaunchScope ls(act ? K_CKPT8_ACT_FWD : K_CKPT8_PACK, n * e * (act ? 2 : 1) + rows * 33.0 * groups_of(cols), 0.0, st);
    if (dtype == AST_F32) launch<float>(true, act, a, rows, cols, st);
    else launch<__nv_bfloat16>(true, act, a, rows, cols, st);
}

void ckpt8_backward(int dtype, int act, const void* codes, const void* exps, const void* dy, size_t lddy, size_t rows, int cols, void* out, size_t ldo,
                    cudaStream_t st) {
    if (!rows) return;
    Args a{};
    a.dy = act ? dy : nullptr; a.lddy = lddy; a.out = out; a.ldo = ldo; a.codes = const_cast<void*>(codes); a.exps = const_cast<void*>(exps);
    const double n = (double)rows * cols, e = dtype == AST_F32 ? 4 : 2;
    LaunchScope ls(act ? K_CKPT8_ACT_BWD : K_CKPT8_UNPACK, n * e * (act ? 2 : 1) + rows * 33.0 * groups_of(cols), 0.0, st);
    if (dtype == AST_F32) launch<float>(false, act, a, rows, cols, st);
    else launch<__nv_bfloat16>(false, act, a, rows, cols, st);
}

}  // namespace ast

// ================================================================================ C ABI
using namespace ast;

namespace {

constexpr size_t MAX_ROWS = ((size_t)1 << 31) - 1, MAX_ELEMS = (size_t)1 << 40;
constexpr int MAX_WIDTH = 65536;

size_t pitch_of(int cols) { return groups_of(cols) * q8::GROUP; }

// sizes of a [rows][cols] tensor with rows `ld` apart
int bad_matrix(const char* what, const void* p, size_t ld, size_t rows, int cols, int dtype) {
    if (!p && rows) return report_error(AST_ERR_ARG, "null argument");
    if (dtype != AST_F32 && dtype != AST_BF16) return report_error(AST_ERR_ARG, "bad dtype");
    if (cols < 1 || rows > MAX_ROWS || (rows && pitch_of(cols) > MAX_ELEMS / rows)) return report_error(AST_ERR_ARG, "rows or columns out of range");
    if (ld < (size_t)cols || (rows && ld > MAX_ELEMS / rows)) return report_error(AST_ERR_ARG, what);
    if (reinterpret_cast<uintptr_t>(p) % (dtype == AST_F32 ? 4 : 2)) return report_error(AST_ERR_ARG, "a tensor does not start at an element of its type");
    return AST_OK;
}
int bad_ckpt(const void* p, size_t rows) {
    if (!p && rows) return report_error(AST_ERR_ARG, "null checkpoint");
    if (reinterpret_cast<uintptr_t>(p) % 16) return report_error(AST_ERR_ARG, "a checkpoint must start at a 16-byte boundary");
    return AST_OK;
}
bool is_act8(int act) { return act == AST_RELU6 || act == AST_RELU || act == AST_SILU || act == AST_GELU; }
char* exps_of(const void* ckpt, size_t rows, int cols) { return const_cast<char*>(static_cast<const char*>(ckpt)) + rows * pitch_of(cols); }
int launched() {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AST_OK : report_error(AST_ERR_CUDA, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

size_t asteroid_ckpt8_bytes(size_t rows, int cols) {
    if (cols < 1 || rows < 1 || rows > MAX_ROWS || pitch_of(cols) > MAX_ELEMS / rows) return 0;
    return rows * (pitch_of(cols) + groups_of(cols));
}

int asteroid_ckpt8_pack(const void* x, size_t ldx, size_t rows, int cols, int dtype, void* ckpt, void* stream) {
    int rc = bad_matrix("ldx out of range", x, ldx, rows, cols, dtype);
    if (rc || (rc = bad_ckpt(ckpt, rows))) return rc;
    ckpt8_forward(dtype, 0, x, ldx, rows, cols, nullptr, 0, ckpt, exps_of(ckpt, rows, cols), (cudaStream_t)stream);
    return launched();
}

int asteroid_ckpt8_unpack(const void* ckpt, size_t rows, int cols, int dtype, void* x, size_t ldx, void* stream) {
    int rc = bad_matrix("ldx out of range", x, ldx, rows, cols, dtype);
    if (rc || (rc = bad_ckpt(ckpt, rows))) return rc;
    ckpt8_backward(dtype, 0, ckpt, exps_of(ckpt, rows, cols), nullptr, 0, rows, cols, x, ldx, (cudaStream_t)stream);
    return launched();
}

int asteroid_ckpt8_act_forward(int act, const void* x, size_t ldx, size_t rows, int cols, int dtype, void* y, size_t ldy, void* ckpt, void* stream) {
    if (!is_act8(act)) return report_error(AST_ERR_ARG, "act must be AST_RELU6, AST_RELU, AST_SILU or AST_GELU");
    int rc = bad_matrix("ldx out of range", x, ldx, rows, cols, dtype);
    if (rc || (rc = bad_matrix("ldy out of range", y, ldy, rows, cols, dtype)) || (rc = bad_ckpt(ckpt, rows))) return rc;
    ckpt8_forward(dtype, act, x, ldx, rows, cols, y, ldy, ckpt, exps_of(ckpt, rows, cols), (cudaStream_t)stream);
    return launched();
}

int asteroid_ckpt8_act_backward(int act, const void* ckpt, const void* dy, size_t lddy, size_t rows, int cols, int dtype, void* dx, size_t lddx,
                                void* stream) {
    if (!is_act8(act)) return report_error(AST_ERR_ARG, "act must be AST_RELU6, AST_RELU, AST_SILU or AST_GELU");
    int rc = bad_matrix("lddy out of range", dy, lddy, rows, cols, dtype);
    if (rc || (rc = bad_matrix("lddx out of range", dx, lddx, rows, cols, dtype)) || (rc = bad_ckpt(ckpt, rows))) return rc;
    ckpt8_backward(dtype, act, ckpt, exps_of(ckpt, rows, cols), dy, lddy, rows, cols, dx, lddx, (cudaStream_t)stream);
    return launched();
}

static int bad_widths(size_t rows, int c_in, int c_out, int dtype) {
    if (dtype != AST_F32 && dtype != AST_BF16) return report_error(AST_ERR_ARG, "bad dtype");
    if (rows > MAX_ROWS || c_in < 1 || c_out < 1 || c_in > MAX_WIDTH || c_out > MAX_WIDTH) return report_error(AST_ERR_ARG, "rows, c_in or c_out out of range");
    return AST_OK;
}

size_t asteroid_ckpt8_linear_wgrad_workspace(size_t rows, int c_in, int c_out, int dtype) {
    if (bad_widths(rows, c_in, c_out, dtype)) return 0;
    return ckpt8_wgrad_most_scratch(dtype, rows, c_in, c_out) * sizeof(float);
}

static int bad_linear_wgrad(const void* ckpt, const void* dy, size_t lddy, size_t rows, int c_in, int c_out, int dtype, const float* dw, const float* db,
                            const void* workspace, size_t workspace_bytes) {
    int rc = bad_widths(rows, c_in, c_out, dtype);
    if (rc || (rc = bad_matrix("lddy out of range", dy, lddy, rows, c_out, dtype)) || (rc = bad_ckpt(ckpt, rows))) return rc;
    if (!dw) return report_error(AST_ERR_ARG, "null argument");
    if ((reinterpret_cast<uintptr_t>(dw) | reinterpret_cast<uintptr_t>(db)) % 4) return report_error(AST_ERR_ARG, "a tensor does not start at an element of its type");
    const size_t need = ckpt8_wgrad_most_scratch(dtype, rows, c_in, c_out) * sizeof(float);
    if (need && (!workspace || workspace_bytes < need)) return report_error(AST_ERR_ARG, "the workspace is too small");
    if (need && reinterpret_cast<uintptr_t>(workspace) % 16) return report_error(AST_ERR_ARG, "a workspace must start at a 16-byte boundary");
    return AST_OK;
}

int asteroid_ckpt8_linear_wgrad(const void* ckpt, const void* dy, size_t lddy, size_t rows, int c_in, int c_out, int dtype, float* dw, float* db,
                                int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = bad_linear_wgrad(ckpt, dy, lddy, rows, c_in, c_out, dtype, dw, db, workspace, workspace_bytes)) return rc;
    ckpt8_wgrad(dtype, ckpt, exps_of(ckpt, rows, c_in), dy, lddy, rows, c_in, c_out, dw, db, accumulate != 0, static_cast<float*>(workspace), nullptr,
                (cudaStream_t)stream);
    return launched();
}

int asteroid_selftest_ckpt8_linear_wgrad(const void* ckpt, const void* dy, size_t lddy, size_t rows, int c_in, int c_out, int dtype, float* dw, float* db,
                                         int accumulate, void* workspace, size_t workspace_bytes, int silent_after) {
    if (int rc = bad_linear_wgrad(ckpt, dy, lddy, rows, c_in, c_out, dtype, dw, db, workspace, workspace_bytes)) return rc;
    const size_t unit = dtype == AST_F32 ? 2 : 8;
    if (silent_after < 0 || rows < 1 || lddy % unit || reinterpret_cast<uintptr_t>(dy) % (unit == 2 ? 8 : 16) || (dtype == AST_F32 && c_out % 2))
        return report_error(AST_ERR_ARG, "the self-test takes rows of dy at 16-byte (float32: 8-byte) boundaries, and a number of steps");
    int *err = nullptr, h = 0;
    cudaError_t e = cudaMalloc((void**)&err, sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(err, 0, sizeof(int));
    if (e == cudaSuccess) {
        ckpt8_wgrad(dtype, ckpt, exps_of(ckpt, rows, c_in), dy, lddy, rows, c_in, c_out, dw, db, accumulate != 0, static_cast<float*>(workspace), err, 0, silent_after);
        e = cudaDeviceSynchronize();
    }
    if (e == cudaSuccess) e = cudaMemcpy(&h, err, sizeof h, cudaMemcpyDeviceToHost);
    cudaFree(err);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) {
        cudaGetLastError();
        return report_error(AST_ERR_CUDA, cudaGetErrorString(e));
    }
    return h ? report_error(AST_ERR_TIMEOUT, "a bounded device-side wait expired (self-test: expected)") : AST_OK;
}

}  // extern "C"
