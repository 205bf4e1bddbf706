// aspis_clip.hip -- gfx950 kernels of the norm, clipping and update
// operators: the global norm of a list of tensors, clipping by it, clipping
// every row of a tensor by its own norm, and the model update that applies
// the clip as it reads the gradient.
//
// All of them stream: a few flops per element, so memory bounds them from
// some megabytes on and launches below that.  Sums of squares are fp64: the
// square of any f32 fits, the sum needs no scaling pass, and the rate
// (a conversion and an fma per element) stays above what memory delivers.
// Every sum is split by sizes alone and joined in a fixed order, without
// atomics, so equal inputs give equal bits wherever they lie.
#include "aspis_clip.h"

#include <cfloat>

namespace aspis {

namespace {

// Sixteen bytes of a tensor.  The address is aligned to the element only;
// gfx950 takes such vector accesses.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
#define GLOBAL __attribute__((address_space(1)))

// ---------------------------------------------------------------------------
// element types: V elements per 16 bytes, to and from f32

struct F32 {
    typedef float T;
    typedef u32x4_at4 Vec;
    static constexpr int V = 4;
    __device__ static float get(T x) { return x; }
    __device__ static T put(float x) { return x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[j]);
        return w;
    }
};

struct BF16 {
    typedef __bf16 T;
    typedef u32x4_at2 Vec;
    static constexpr int V = 8;
    __device__ static float get(T x) { return (float)x; }
    __device__ static T put(float x) { return (__bf16)x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = __builtin_bit_cast(
                uint32_t, __builtin_convertvector((f32x2){x[2 * j], x[2 * j + 1]}, b2));
        return w;
    }
};

struct F16 {
    typedef _Float16 T;
    typedef u32x4_at2 Vec;
    static constexpr int V = 8;
    __device__ static float get(T x) { return (float)x; }
    __device__ static T put(float x) { return (_Float16)x; }
    __device__ static void unpack(u32x4 w, float (&x)[V]) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t word = w[j];   // (a bit cast of w[j] itself reads w[0])
            const h2 h = __builtin_bit_cast(h2, word);
            x[2 * j] = (float)h[0];
            x[2 * j + 1] = (float)h[1];
        }
    }
    __device__ static u32x4 pack(const float (&x)[V]) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = __builtin_bit_cast(
                uint32_t, __builtin_convertvector((f32x2){x[2 * j], x[2 * j + 1]}, h2));
        return w;
    }
};

template <typename E>
using Ptr = const typename E::T GLOBAL *;
template <typename E>
using MutPtr = typename E::T GLOBAL *;

template <typename E>
__device__ __forceinline__ u32x4 load_vec(Ptr<E> p) {
    return *(const typename E::Vec GLOBAL *)p;
}
template <typename E>
__device__ __forceinline__ void store_vec(MutPtr<E> p, u32x4 v) {
    *(typename E::Vec GLOBAL *)p = v;
}

// Calls f with the element type of a dtype code (uniform over the workgroup).
template <typename F>
__device__ __forceinline__ void with_type(int dtype, F &&f) {
    if (dtype == ASPIS_F32) f(F32());
    else if (dtype == ASPIS_BF16) f(BF16());
    else f(F16());
}

// ---------------------------------------------------------------------------
// sums

// Over groups of L consecutive lanes (a power of two <= 64), to every lane.
// Each step adds the same two values on both sides, so all lanes agree.
template <int L>
__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// Over the workgroup of B threads, to every thread.  Two barriers: the
// second lets the caller use it again at once.
template <int B>
__device__ __forceinline__ double block_sum(double v) {
    v = lanes_sum<64>(v);
    if constexpr (B == 64) return v;
    __shared__ double part[B / 64];
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    double s = part[0];
#pragma unroll
    for (int w = 1; w < B / 64; ++w) s += part[w];
    __syncthreads();
    return s;
}

// The sum of n values in memory, thread t taking t, t + B, ...
template <int B>
__device__ __forceinline__ double block_sum_of(const double *p, int n) {
    double v = 0.0;
    for (int i = threadIdx.x; i < n; i += B) v += p[i];
    return block_sum<B>(v);
}

__device__ __forceinline__ double add_square(float x, double acc) {
    const double d = (double)x;
    return __builtin_fma(d, d, acc);
}

template <typename E>
__device__ __forceinline__ void add_squares(u32x4 w, double (&acc)[2]) {
    float x[E::V];
    E::unpack(w, x);
#pragma unroll
    for (int j = 0; j < E::V; ++j) acc[j & 1] = add_square(x[j], acc[j & 1]);
}

// Adds the squares of n elements, split over the B threads of a workgroup.
template <typename E, int B, int U>
__device__ __forceinline__ void span_squares(Ptr<E> p, int n, double (&acc)[2]) {
    const int nv = n / E::V;
    int i = threadIdx.x;
    for (; i + (U - 1) * B < nv; i += U * B) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_vec<E>(p + (int64_t)(i + u * B) * E::V);
#pragma unroll
        for (int u = 0; u < U; ++u) add_squares<E>(w[u], acc);
    }
    for (; i < nv; i += B) add_squares<E>(load_vec<E>(p + (int64_t)i * E::V), acc);
    const int rest = nv * E::V + threadIdx.x;
    if (rest < n) acc[0] = add_square(E::get(p[rest]), acc[0]);
}

// ---------------------------------------------------------------------------
// the coefficient

// c = m * 2^e with m in [1/2, 1), or m = c = 1, e = 0: x * m neither
// overflows nor, for e = 0, loses bits, and c may be far below the smallest
// f32 (a norm of 1e40 with a bound of 1).
struct Coef {
    float m;
    int e;
    __device__ float operator()(float x) const { return __builtin_amdgcn_ldexpf(x * m, e); }
    __device__ bool one() const { return m == 1.0f; }
};

__device__ __forceinline__ Coef coefficient(double sumsq, double max_norm) {
    const double norm = sqrt(sumsq);
    if (norm <= max_norm || max_norm > DBL_MAX) return {1.0f, 0};
    const double c = max_norm / norm;
    int e = 0;
    const float m = (float)frexp(c, &e);
    // rounding may carry m to 1: the same value, one exponent up
    if (m == 1.0f) return {0.5f, e + 1};
    return {m, e};
}

// The global norm's sum, from the partial sums (every workgroup adds them
// in the same order) or as given; workgroup 0 writes it down.
template <int B>
__device__ __forceinline__ double take_sumsq(const NormIn &in) {
    double s;
    if (in.n_partial > 0) {
        s = block_sum_of<B>(in.partial, in.n_partial);
        if (blockIdx.x == 0 && threadIdx.x == 0) *in.sumsq = s;
    } else {
        s = *in.sumsq;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *in.norm = (float)sqrt(s);
    return s;
}

// out = c * x over n elements, split over the B threads of a workgroup; out
// may be x.
template <typename E, int B, int U>
__device__ __forceinline__ void span_scale(Ptr<E> p, MutPtr<E> o, int n, Coef c) {
    const int nv = n / E::V;
    auto scaled = [&](u32x4 w) {
        float x[E::V];
        E::unpack(w, x);
#pragma unroll
        for (int j = 0; j < E::V; ++j) x[j] = c(x[j]);
        return E::pack(x);
    };
    int i = threadIdx.x;
    for (; i + (U - 1) * B < nv; i += U * B) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_vec<E>(p + (int64_t)(i + u * B) * E::V);
#pragma unroll
        for (int u = 0; u < U; ++u)
            store_vec<E>(o + (int64_t)(i + u * B) * E::V, scaled(w[u]));
    }
    for (; i < nv; i += B)
        store_vec<E>(o + (int64_t)i * E::V, scaled(load_vec<E>(p + (int64_t)i * E::V)));
    const int rest = nv * E::V + threadIdx.x;
    if (rest < n) o[rest] = E::put(c(E::get(p[rest])));
}

// ---------------------------------------------------------------------------
// lists of tensors

constexpr int kListBlock = 256;

__global__ __launch_bounds__(kListBlock) void
list_sumsq_kernel(const aspis_chunk *__restrict__ table, int64_t n_chunks, double *partial,
                  double *chunk_sums) {
    double acc[2] = {0.0, 0.0};
    double total = 0.0;
    for (int64_t k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const aspis_chunk c = table[k];
        with_type(c.info, [&](auto e) {
            typedef decltype(e) E;
            span_squares<E, kListBlock, 4>((Ptr<E>)c.addr, c.n, acc);
        });
        if (chunk_sums != nullptr) {
            const double s = block_sum<kListBlock>(acc[0] + acc[1]);
            if (threadIdx.x == 0) chunk_sums[k] = s;
            total += s;
            acc[0] = acc[1] = 0.0;
        }
    }
    if (chunk_sums == nullptr) total = block_sum<kListBlock>(acc[0] + acc[1]);
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

// Workgroup 0 joins the partial sums; the others, one wave per tensor, the
// tensors' own chunk sums.
__global__ __launch_bounds__(kListBlock) void
list_norm_kernel(const aspis_chunk *__restrict__ tensors, int32_t n_tensors, NormIn in,
                 const double *__restrict__ chunk_sums, float *each) {
    if (blockIdx.x == 0) {
        if (in.n_partial > 0) {
            take_sumsq<kListBlock>(in);
        } else if (threadIdx.x == 0) {   // an empty list
            *in.sumsq = 0.0;
            *in.norm = 0.0f;
        }
        return;
    }
    const int t = (blockIdx.x - 1) * (kListBlock / 64) + threadIdx.x / 64;
    if (t >= n_tensors) return;
    const aspis_chunk c = tensors[t];
    double v = 0.0;
    for (int i = threadIdx.x % 64; i < c.n; i += 64) v += chunk_sums[c.addr + i];
    v = lanes_sum<64>(v);
    if (threadIdx.x % 64 == 0) each[t] = (float)sqrt(v);
}

__global__ __launch_bounds__(kListBlock) void
list_scale_kernel(const aspis_chunk *__restrict__ table, const aspis_chunk *__restrict__ out,
                  int64_t n_chunks, NormIn in) {
    const Coef coef = coefficient(take_sumsq<kListBlock>(in), in.max_norm);
    if (out == nullptr && coef.one()) return;   // in place: already there
    for (int64_t k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const aspis_chunk c = table[k];
        const uint64_t to = out != nullptr ? out[k].addr : c.addr;
        with_type(c.info, [&](auto e) {
            typedef decltype(e) E;
            span_scale<E, kListBlock, 4>((Ptr<E>)c.addr, (MutPtr<E>)to, c.n, coef);
        });
    }
}

// ---------------------------------------------------------------------------
// the updates: four elements per lane and step, so that the f32 tensors move
// 16 bytes and 16-bit ones 8

__device__ __forceinline__ void load_four(uint64_t addr, int dtype, int64_t i, float (&x)[4]) {
    if (dtype == ASPIS_F32) {
        F32::unpack(load_vec<F32>((Ptr<F32>)addr + i), x);
        return;
    }
    const u32x2 w = *(const u32x2_at2 GLOBAL *)((const uint16_t GLOBAL *)addr + i);
    float y[8];
    if (dtype == ASPIS_BF16) BF16::unpack((u32x4){w.x, w.y, 0, 0}, y);
    else F16::unpack((u32x4){w.x, w.y, 0, 0}, y);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j];
}

__device__ __forceinline__ void store_four(uint64_t addr, int dtype, int64_t i,
                                           const float (&x)[4]) {
    if (dtype == ASPIS_F32) {
        store_vec<F32>((MutPtr<F32>)addr + i, F32::pack(x));
        return;
    }
    const float y[8] = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    const u32x4 w = dtype == ASPIS_BF16 ? BF16::pack(y) : F16::pack(y);
    *(u32x2_at2 GLOBAL *)((uint16_t GLOBAL *)addr + i) = (u32x2){w.x, w.y};
}

__device__ __forceinline__ float load_one(uint64_t addr, int dtype, int64_t i) {
    float x = 0.0f;
    with_type(dtype, [&](auto e) { x = decltype(e)::get(((Ptr<decltype(e)>)addr)[i]); });
    return x;
}
__device__ __forceinline__ void store_one(uint64_t addr, int dtype, int64_t i, float x) {
    with_type(dtype, [&](auto e) {
        ((MutPtr<decltype(e)>)addr)[i] = decltype(e)::put(x);
    });
}

// The state of one element besides its parameter: S tensors.
struct Sgd {
    static constexpr int S = 1;
    SgdArgs a;
    __device__ void operator()(float g, float &p, float (&s)[S]) const {
        if (a.decay != 0.0f) g = fmaf(a.decay, p, g);
        s[0] = fmaf(a.momentum, s[0], g);
        const float d = a.nesterov ? fmaf(a.momentum, s[0], g) : s[0];
        p = fmaf(-a.lr, d, p);
    }
};
struct PlainSgd {
    static constexpr int S = 0;
    SgdArgs a;
    __device__ void operator()(float g, float &p, float (&)[1]) const {
        if (a.decay != 0.0f) g = fmaf(a.decay, p, g);
        p = fmaf(-a.lr, g, p);
    }
};
struct AdamW {
    static constexpr int S = 2;
    AdamArgs a;
    __device__ void operator()(float g, float &p, float (&s)[S]) const {
        s[0] = fmaf(a.beta1, s[0], a.rest1 * g);
        s[1] = fmaf(a.beta2, s[1], a.rest2 * g * g);
        const float root = fmaf(sqrtf(s[1]), a.root2, a.eps);
        p = fmaf(-a.step_size, s[0] / root, p * a.shrink);
    }
};

struct UpdateTables {
    const aspis_chunk *params, *grads, *state[2], *copies;
};

template <typename Rule>
__global__ __launch_bounds__(kListBlock) void
update_kernel(UpdateTables t, int64_t n_chunks, NormIn in, Rule rule, bool skip) {
    constexpr int S = Rule::S, W = S > 0 ? S : 1;
    const double sumsq = take_sumsq<kListBlock>(in);
    if (skip && !(sumsq <= DBL_MAX)) return;
    const Coef coef = coefficient(sumsq, in.max_norm);
    for (int64_t k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const aspis_chunk g = t.grads[k];
        const uint64_t pa = t.params[k].addr;
        uint64_t sa[W] = {};
#pragma unroll
        for (int j = 0; j < S; ++j) sa[j] = t.state[j][k].addr;
        const aspis_chunk copy = t.copies != nullptr ? t.copies[k] : aspis_chunk{0, 0, 0};
        const int nv = g.n / 4;
        for (int i = threadIdx.x; i < nv; i += kListBlock) {
            const int64_t at = (int64_t)i * 4;
            float x[4], p[4], s[W][4];
            load_four(g.addr, g.info, at, x);
            load_four(pa, ASPIS_F32, at, p);
#pragma unroll
            for (int j = 0; j < S; ++j) load_four(sa[j], ASPIS_F32, at, s[j]);
#pragma unroll
            for (int l = 0; l < 4; ++l) {
                float one[W];
#pragma unroll
                for (int j = 0; j < S; ++j) one[j] = s[j][l];
                rule(coef(x[l]), p[l], one);
#pragma unroll
                for (int j = 0; j < S; ++j) s[j][l] = one[j];
            }
            store_four(pa, ASPIS_F32, at, p);
#pragma unroll
            for (int j = 0; j < S; ++j) store_four(sa[j], ASPIS_F32, at, s[j]);
            if (copy.n > 0) store_four(copy.addr, copy.info, at, p);
        }
        const int i = nv * 4 + threadIdx.x;
        if (i < g.n) {
            float one[W], p = load_one(pa, ASPIS_F32, i);
#pragma unroll
            for (int j = 0; j < S; ++j) one[j] = load_one(sa[j], ASPIS_F32, i);
            rule(coef(load_one(g.addr, g.info, i)), p, one);
            store_one(pa, ASPIS_F32, i, p);
#pragma unroll
            for (int j = 0; j < S; ++j) store_one(sa[j], ASPIS_F32, i, one[j]);
            if (copy.n > 0) store_one(copy.addr, copy.info, i, p);
        }
    }
}

// ---------------------------------------------------------------------------
// rows

// A row in the registers of L lanes, R vectors each: read once, its norm,
// written once.  L <= 64: B / L rows per workgroup; L == B: one.
template <typename E, int L, int B, int R>
__global__ __launch_bounds__(B) void row_kernel(RowArgs a) {
    constexpr int V = E::V, G = B / L;
    const int lane = threadIdx.x % L;
    for (int64_t row0 = (int64_t)blockIdx.x * G; row0 < a.rows; row0 += (int64_t)gridDim.x * G) {
        const int64_t row = row0 + threadIdx.x / L;
        const int d = row < a.rows ? (int)a.d : 0;
        const Ptr<E> p = (Ptr<E>)a.x + row * a.ld;
        u32x4 w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = (lane + r * L) * V;
            w[r] = (u32x4){0, 0, 0, 0};
            if (i + V <= d) {
                w[r] = load_vec<E>(p + i);
            } else if (i < d) {
                float x[V];
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = i + j < d ? E::get(p[i + j]) : 0.0f;
                w[r] = E::pack(x);
            }
        }
        double acc[2] = {0.0, 0.0};
#pragma unroll
        for (int r = 0; r < R; ++r) add_squares<E>(w[r], acc);
        double s;
        if constexpr (L == B) s = block_sum<B>(acc[0] + acc[1]);
        else s = lanes_sum<L>(acc[0] + acc[1]);
        if (d > 0 && lane == 0 && a.norms != nullptr) a.norms[row] = (float)sqrt(s);
        if (a.out == nullptr) continue;
        const Coef c = coefficient(s, a.max_norm);
        if (a.out == a.x && c.one()) continue;
        const MutPtr<E> o = (MutPtr<E>)a.out + row * a.ldo;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = (lane + r * L) * V;
            float x[V];
            E::unpack(w[r], x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = c(x[j]);
            if (i + V <= d) {
                store_vec<E>(o + i, E::pack(x));
            } else if (i < d) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (i + j < d) o[i + j] = E::put(x[j]);
            }
        }
    }
}

__global__ __launch_bounds__(kListBlock) void empty_rows_kernel(float *norms, int64_t rows) {
    for (int64_t i = blockIdx.x * (int64_t)kListBlock + threadIdx.x; i < rows;
         i += (int64_t)gridDim.x * kListBlock)
        norms[i] = 0.0f;
}

// Segments of long rows.  One launch scales the segments of rows
// [scale0, scale0 + n_scale) whose sums are there, and sums those of rows
// [sum0, sum0 + n_sum); the two kinds of work alternate over the workgroups.
struct SegArgs {
    RowArgs a;
    int64_t seg;
    int32_t parts;
    int64_t scale0, sum0;
    int64_t n_scale, n_sum;   // segments
};

template <typename E>
__global__ __launch_bounds__(kListBlock) void segment_kernel(SegArgs g) {
    const int64_t both = g.n_scale < g.n_sum ? g.n_scale : g.n_sum;
    const int64_t b = blockIdx.x;
    bool scale;
    int64_t item;
    if (b < 2 * both) {
        scale = (b & 1) != 0;
        item = b >> 1;
    } else {
        scale = g.n_scale > g.n_sum;
        item = b - both;
    }
    const int64_t row = (scale ? g.scale0 : g.sum0) + item / g.parts;
    const int part = (int)(item % g.parts);
    const int64_t first = part * g.seg;
    const int n = (int)(g.a.d - first < g.seg ? g.a.d - first : g.seg);
    const Ptr<E> p = (Ptr<E>)g.a.x + row * g.a.ld + first;
    double *sums = g.a.partial + row * g.parts;
    if (!scale) {
        double acc[2] = {0.0, 0.0};
        span_squares<E, kListBlock, 4>(p, n, acc);
        const double s = block_sum<kListBlock>(acc[0] + acc[1]);
        if (threadIdx.x == 0) sums[part] = s;
        return;
    }
    const double s = block_sum_of<kListBlock>(sums, g.parts);
    if (part == 0 && threadIdx.x == 0 && g.a.norms != nullptr) g.a.norms[row] = (float)sqrt(s);
    const Coef c = coefficient(s, g.a.max_norm);
    if (g.a.out == g.a.x && c.one()) return;
    span_scale<E, kListBlock, 4>(p, (MutPtr<E>)g.a.out + row * g.a.ldo + first, n, c);
}

// The norms alone of long rows, from their segments' sums.
__global__ __launch_bounds__(kListBlock) void segment_norm_kernel(const double *sums, int parts,
                                                                  float *norms) {
    const double s = block_sum_of<kListBlock>(sums + (int64_t)blockIdx.x * parts, parts);
    if (threadIdx.x == 0) norms[blockIdx.x] = (float)sqrt(s);
}

template <typename E, int L, int B, int R>
void start_rows(const RowArgs &a, hipStream_t s) {
    const int64_t blocks = (a.rows + B / L - 1) / (B / L);
    const int64_t cap = 1 << 20;
    row_kernel<E, L, B, R><<<(unsigned)(blocks < cap ? blocks : cap), B, 0, s>>>(a);
}

template <typename E>
hipError_t rows_of(const RowArgs &a, hipStream_t s) {
    const int64_t nv = (a.d + E::V - 1) / E::V;
    if (nv <= kRowVecs) {
        if (nv <= 4) start_rows<E, 4, 256, 1>(a, s);
        else if (nv <= 16) start_rows<E, 16, 256, 1>(a, s);
        else if (nv <= 64) start_rows<E, 64, 256, 1>(a, s);
        else if (nv <= 128) start_rows<E, 64, 256, 2>(a, s);
        else if (nv <= 256) start_rows<E, 64, 256, 4>(a, s);
        else if (nv <= 512) start_rows<E, 256, 256, 2>(a, s);
        else if (nv <= 1024) start_rows<E, 256, 256, 4>(a, s);
        else if (nv <= 2048) start_rows<E, 256, 256, 8>(a, s);
        else if (nv <= 4096) start_rows<E, 1024, 1024, 4>(a, s);
        else start_rows<E, 1024, 1024, 8>(a, s);
        return hipGetLastError();
    }
    const RowSplit split = row_split(a.d, (int)sizeof(typename E::T));
    // rows per launch: what stays in the last-level cache until the next
    // launch scales it
    const int64_t bytes = a.d * (int64_t)sizeof(typename E::T);
    int64_t step = (int64_t)(64 << 20) / bytes;
    if (step < 1) step = 1;
    if (a.out == nullptr) step = a.rows;
    while (step * split.parts > (1 << 20) && step > 1) step = (step + 1) / 2;
    for (int64_t r = 0; r < a.rows + (a.out != nullptr ? step : 0); r += step) {
        SegArgs g{};
        g.a = a;
        g.seg = split.seg;
        g.parts = split.parts;
        g.sum0 = r;
        const int64_t sum_rows = r < a.rows ? (a.rows - r < step ? a.rows - r : step) : 0;
        g.n_sum = sum_rows * split.parts;
        if (a.out != nullptr && r > 0) {
            g.scale0 = r - step;
            g.n_scale = (a.rows - g.scale0 < step ? a.rows - g.scale0 : step) * split.parts;
        }
        if (g.n_sum + g.n_scale == 0) continue;
        segment_kernel<E><<<(unsigned)(g.n_sum + g.n_scale), kListBlock, 0, s>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.out == nullptr)
        segment_norm_kernel<<<(unsigned)a.rows, kListBlock, 0, s>>>(a.partial, split.parts,
                                                                    a.norms);
    return hipGetLastError();
}

unsigned list_grid(int64_t n_chunks) { return n_chunks > 0 ? (unsigned)norm_groups(n_chunks) : 1u; }

}  // namespace

hipError_t launch_list_sumsq(const aspis_chunk *table, int64_t n_chunks, double *partial,
                             double *chunk_sums, hipStream_t s) {
    list_sumsq_kernel<<<list_grid(n_chunks), kListBlock, 0, s>>>(table, n_chunks, partial,
                                                                 chunk_sums);
    return hipGetLastError();
}

hipError_t launch_list_norm(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors,
                            const NormIn &in, const double *chunk_sums, float *each,
                            hipStream_t s) {
    const int waves = kListBlock / 64;
    const unsigned grid = 1u + (each != nullptr ? (unsigned)((n_tensors + waves - 1) / waves) : 0u);
    list_norm_kernel<<<grid, kListBlock, 0, s>>>(table + n_chunks, n_tensors, in, chunk_sums,
                                                 each);
    return hipGetLastError();
}

hipError_t launch_list_scale(const aspis_chunk *table, const aspis_chunk *out, int64_t n_chunks,
                             const NormIn &in, hipStream_t s) {
    list_scale_kernel<<<list_grid(n_chunks), kListBlock, 0, s>>>(table, out, n_chunks, in);
    return hipGetLastError();
}

hipError_t launch_sgd(const aspis_chunk *params, const aspis_chunk *grads,
                      const aspis_chunk *mean, const aspis_chunk *copies, int64_t n_chunks,
                      const NormIn &in, const SgdArgs &a, bool skip, hipStream_t s) {
    const UpdateTables t{params, grads, {mean, nullptr}, copies};
    if (mean != nullptr)
        update_kernel<<<list_grid(n_chunks), kListBlock, 0, s>>>(t, n_chunks, in, Sgd{a}, skip);
    else
        update_kernel<<<list_grid(n_chunks), kListBlock, 0, s>>>(t, n_chunks, in, PlainSgd{a},
                                                                 skip);
    return hipGetLastError();
}

hipError_t launch_adamw(const aspis_chunk *params, const aspis_chunk *grads,
                        const aspis_chunk *mean, const aspis_chunk *square,
                        const aspis_chunk *copies, int64_t n_chunks, const NormIn &in,
                        const AdamArgs &a, bool skip, hipStream_t s) {
    const UpdateTables t{params, grads, {mean, square}, copies};
    update_kernel<<<list_grid(n_chunks), kListBlock, 0, s>>>(t, n_chunks, in, AdamW{a}, skip);
    return hipGetLastError();
}

hipError_t launch_rows(const RowArgs &a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    if (a.d == 0) {
        if (a.norms == nullptr) return hipSuccess;
        const int64_t blocks = (a.rows + kListBlock - 1) / kListBlock;
        empty_rows_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), kListBlock, 0, s>>>(
            a.norms, a.rows);
        return hipGetLastError();
    }
    if (a.dtype == ASPIS_F32) return rows_of<F32>(a, s);
    if (a.dtype == ASPIS_BF16) return rows_of<BF16>(a, s);
    return rows_of<F16>(a, s);
}

}  // namespace aspis
