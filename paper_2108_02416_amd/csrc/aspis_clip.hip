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
// atomics, so equal inputs give equal bits wherever they lie.  A list's order
// is the same in every call, whichever kernels do it: a chunk's 256 threads,
// a norm workgroup's chunks thread by thread, its lanes, its waves one after
// the other, then the workgroups (block_sum_of).
#include "aspis_clip.h"

#include <atomic>
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

// Once: the data is not needed again soon (non-temporal).
enum class Use { Again, Once };

template <typename E, Use USE = Use::Again>
__device__ __forceinline__ u32x4 load_vec(Ptr<E> p) {
    const typename E::Vec GLOBAL *q = (const typename E::Vec GLOBAL *)p;
    if constexpr (USE == Use::Once) return __builtin_nontemporal_load(q);
    return *q;
}
template <typename E, Use USE = Use::Again>
__device__ __forceinline__ void store_vec(MutPtr<E> p, u32x4 v) {
    typename E::Vec GLOBAL *q = (typename E::Vec GLOBAL *)p;
    if constexpr (USE == Use::Once) __builtin_nontemporal_store((typename E::Vec)v, q);
    else *q = v;
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

// v of the lane that the DPP control names.
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)w, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(w >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Over groups of L consecutive lanes (a power of two <= 64), to every lane.
// Both partners of a step add the same two values, so all lanes agree.  Up
// to 16 lanes by DPP: within quads, then the mirrors pair the quads.
template <int L>
__device__ __forceinline__ double lanes_sum(double v) {
    if constexpr (L >= 2) v += dpp<0xB1>(v);    // quad_perm 1,0,3,2
    if constexpr (L >= 4) v += dpp<0x4E>(v);    // quad_perm 2,3,0,1
    if constexpr (L >= 8) v += dpp<0x141>(v);   // row_half_mirror
    if constexpr (L >= 16) v += dpp<0x140>(v);  // row_mirror
    if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (L >= 64) v += __shfl_xor(v, 32, 64);
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

// The sum of n values in memory, thread t of the first 256 taking t, t + 256,
// ...: the same in a workgroup of any size.
template <int B>
__device__ __forceinline__ double block_sum_of(const double *p, int n) {
    static_assert(B >= 256, "256 threads share the sum");
    double v = 0.0;
    if (threadIdx.x < 256)
        for (int i = threadIdx.x; i < n; i += 256) v += p[i];
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

// ---------------------------------------------------------------------------
// elements in registers

// n elements in the registers of L lanes: vectors lane, lane + L, ..., R at
// most, and of the n % V elements after the last whole vector, elements lane,
// lane + L, ...; zeros past the end.
template <typename E, int L, int R>
struct Span {
    static constexpr int V = E::V, Q = (V - 2 + L) / L;
    // 16-bit elements at an address that is not a multiple of four: a 16-byte
    // load there takes the memory pipeline longer, so the vectors are loaded
    // from one element earlier (in the same aligned word as the first
    // element, which is never the first of an allocation) and shifted, the
    // last element coming from the next lane.  6,900 rows of 10,007 f16: 50.8
    // against 54.4 us; a list of 200M bf16 from an odd place: clip 203 against
    // 218 us.  Not in a wave's rows (50,000 of 1,001: 37.7 against 36.0) nor
    // with more vectors (24: the registers spill).
    static constexpr bool kShift = V == 8 && L >= 256 && R >= 2 && R <= 8;
    u32x4 w[R];
    typename E::T tail[Q];

    template <Use USE>
    __device__ __forceinline__ void load(Ptr<E> p, int n, int lane) {
        const bool odd = kShift && ((uint64_t)p & 2) != 0;
        const Ptr<E> from = odd ? p - 1 : p;
        const int nv = n / V;
        if (n == R * L * V) {
#pragma unroll
            for (int r = 0; r < R; ++r) w[r] = load_vec<E, USE>(from + (lane + r * L) * V);
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                w[r] = (u32x4){0, 0, 0, 0};
                if (lane + r * L < nv) w[r] = load_vec<E, USE>(from + (lane + r * L) * V);
            }
        }
        if constexpr (kShift)
            if (odd) {
                uint32_t own[R];   // where the next lane does not load the next vector
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    own[r] = 0;
                    const int i = lane + r * L;
                    if (i < nv && (lane == L - 1 || threadIdx.x % 64 == 63 || i == nv - 1))
                        own[r] = *(const uint16_t GLOBAL *)(p + i * V + 7);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int i = lane + r * L;
                    const u32x4 a = w[r];
                    uint32_t last = __builtin_amdgcn_update_dpp(0, (int)a.x, 0x130, 0xF, 0xF, true);
                    if (lane == L - 1 || threadIdx.x % 64 == 63 || i == nv - 1) last = own[r];
                    if (i < nv)
                        w[r] = (u32x4){__builtin_amdgcn_alignbit(a.y, a.x, 16),
                                       __builtin_amdgcn_alignbit(a.z, a.y, 16),
                                       __builtin_amdgcn_alignbit(a.w, a.z, 16),
                                       last << 16 | a.w >> 16};
                }
            }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int i = nv * V + lane + q * L;
            tail[q] = i < n ? p[i] : typename E::T(0);
        }
    }
    // Adds the squares to two sums, vector after vector: spans one behind the
    // other add up as one long span does.
    __device__ __forceinline__ void squares(double (&acc)[2]) const {
#pragma unroll
        for (int r = 0; r < R; ++r) add_squares<E>(w[r], acc);
#pragma unroll
        for (int q = 0; q < Q; ++q) acc[q & 1] = add_square(E::get(tail[q]), acc[q & 1]);
    }
    __device__ __forceinline__ double squares() const {
        double acc[2] = {0.0, 0.0};
        squares(acc);
        return acc[0] + acc[1];
    }
    // Writes c times the elements, their own bits for c = 1 (a product would
    // turn a signalling NaN into a quiet one); o may be where they came from.
    template <Use USE>
    __device__ __forceinline__ void store(MutPtr<E> o, int n, int lane, Coef c) const {
        const int nv = n / V;
        const bool same = c.one();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (n != R * L * V && lane + r * L >= nv) continue;
            // unpacked anew: kept from squares() on, 16-bit elements would
            // take twice the registers
            u32x4 v = w[r];
            if constexpr (V == 8) asm volatile("" : "+v"(v));
            if (!same) {
                float x[V];
                E::unpack(v, x);
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = c(x[j]);
                v = E::pack(x);
            }
            store_vec<E, USE>(o + (lane + r * L) * V, v);
        }
        if (n == R * L * V) return;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int i = nv * V + lane + q * L;
            if (i < n) o[i] = same ? tail[q] : E::put(c(E::get(tail[q])));
        }
    }
};
// A chunk in the registers of 256 threads.
template <typename E>
using Tile = Span<E, 256, kChunk / E::V / 256>;

// ---------------------------------------------------------------------------
// the global norm

// Whether the norm as it is written down, in f32, is finite.
__device__ __forceinline__ bool norm_is_finite(double sumsq) {
    return (float)sqrt(sumsq) <= FLT_MAX;
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

// ---------------------------------------------------------------------------
// lists of tensors

constexpr int kListBlock = 256;

__device__ __forceinline__ int chunk_type(const aspis_chunk &c) { return c.info & 3; }
__device__ __forceinline__ int chunk_tensor(const aspis_chunk &c) { return c.info >> 2; }

// The squares of a chunk, split over 256 threads.
template <Use USE>
__device__ __forceinline__ double chunk_squares(const aspis_chunk &c, int t) {
    double s = 0.0;
    with_type(chunk_type(c), [&](auto e) {
        typedef decltype(e) E;
        Tile<E> tile;
        tile.template load<USE>((Ptr<E>)c.addr, c.n, t);
        s = tile.squares();
    });
    return s;
}

// The norm pass: a fixed number of workgroups over groups of `group` chunks
// in turn, one partial sum each.  Chunks from `keep` on are read to stay in
// the last-level cache for the pass that follows.  runs, when not NULL,
// receives the sum of every run of one tensor's chunks in a group, at the
// group's index plus the tensor's: of two runs one after the other at least
// one index is one up, so no two share a place.
// Memory bounds it: 871M mixed elements (1.74 GB) in 257 to 264 us, 6.6 to
// 6.8 TB/s of the 7.1 that a linear read reaches, with
// all of a chunk's 16-byte loads in flight before the first square and the
// next chunk's entry already there; each byte is read once.
__global__ __launch_bounds__(kListBlock) void
list_sumsq_kernel(const aspis_chunk *__restrict__ table, int64_t n_chunks, int group,
                  int64_t keep, double *partial, double *runs) {
    double total = 0.0, run = 0.0;
    int64_t first = (int64_t)blockIdx.x * group, k = first;
    aspis_chunk next = table[k];
    while (k < n_chunks) {
        const aspis_chunk c = next;
        const int64_t now = k, now_first = first;
        if (++k == first + group || k >= n_chunks) k = first += (int64_t)gridDim.x * group;
        next = table[k < n_chunks ? k : now];
        const double squares = now < keep ? chunk_squares<Use::Once>(c, threadIdx.x)
                                          : chunk_squares<Use::Again>(c, threadIdx.x);
        total += squares;
        if (runs == nullptr) continue;
        run += squares;
        if (first != now_first || chunk_tensor(next) != chunk_tensor(c)) {
            const double s = block_sum<kListBlock>(run);
            if (threadIdx.x == 0) runs[now_first / group + chunk_tensor(c)] = s;
            run = 0.0;
        }
    }
    total = block_sum<kListBlock>(total);
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

// Workgroup 0 joins the partial sums, workgroup 1 + t the runs of tensor t:
// 2.2 us for a thousand partial sums, the latency of loads and barriers.
__global__ __launch_bounds__(kListBlock) void
list_norm_kernel(const aspis_chunk *__restrict__ tensors, int group, NormIn in,
                 const double *__restrict__ runs, float *each) {
    if (blockIdx.x == 0) {
        take_sumsq<kListBlock>(in);
        return;
    }
    const aspis_chunk c = tensors[blockIdx.x - 1];
    double s = 0.0;
    if (c.n > 0) {
        const int64_t first = (int64_t)c.addr / group, last = ((int64_t)c.addr + c.n - 1) / group;
        s = block_sum_of<kListBlock>(runs + first + c.info, (int)(last - first) + 1);
    }
    if (threadIdx.x == 0) each[blockIdx.x - 1] = (float)sqrt(s);
}

// One chunk per workgroup, the last first where the list is longer than
// what the cache keeps of it.  The chunk is on its way while the
// coefficient is worked out, unless that may make it unnecessary.
// Memory bounds it: 871M mixed elements read and written in 553 to 560 us, 6.3 TB/s
// (what the norm pass left in the last-level cache included).
__global__ __launch_bounds__(kListBlock) void
list_scale_kernel(const aspis_chunk *__restrict__ table, const aspis_chunk *__restrict__ out,
                  int64_t first, int64_t step, NormIn in) {
    const int64_t k = first + step * blockIdx.x;
    const aspis_chunk c = table[k];
    const uint64_t to = out != nullptr ? out[k].addr : c.addr;
    if (out == nullptr) {
        const Coef coef = coefficient(take_sumsq<kListBlock>(in), in.max_norm);
        if (coef.one()) return;   // in place: already there
        with_type(chunk_type(c), [&](auto e) {
            typedef decltype(e) E;
            Tile<E> tile;
            tile.template load<Use::Once>((Ptr<E>)c.addr, c.n, threadIdx.x);
            tile.template store<Use::Once>((MutPtr<E>)to, c.n, threadIdx.x, coef);
        });
        return;
    }
    with_type(chunk_type(c), [&](auto e) {
        typedef decltype(e) E;
        Tile<E> tile;
        tile.template load<Use::Once>((Ptr<E>)c.addr, c.n, threadIdx.x);
        const Coef coef = coefficient(take_sumsq<kListBlock>(in), in.max_norm);
        tile.template store<Use::Once>((MutPtr<E>)to, c.n, threadIdx.x, coef);
    });
}

// ---------------------------------------------------------------------------
// the updates: four elements per lane, so that the f32 tensors move 16 bytes
// and 16-bit ones 8

template <Use USE>
__device__ __forceinline__ void load_four(uint64_t addr, int dtype, int i, float (&x)[4]) {
    if (dtype == ASPIS_F32) {
        F32::unpack(load_vec<F32, USE>((Ptr<F32>)addr + i), x);
        return;
    }
    const u32x2_at2 GLOBAL *q = (const u32x2_at2 GLOBAL *)((const uint16_t GLOBAL *)addr + i);
    const u32x2 w = USE == Use::Once ? (u32x2)__builtin_nontemporal_load(q) : (u32x2)*q;
    float y[8];
    if (dtype == ASPIS_BF16) BF16::unpack((u32x4){w.x, w.y, 0, 0}, y);
    else F16::unpack((u32x4){w.x, w.y, 0, 0}, y);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j];
}

template <Use USE>
__device__ __forceinline__ void store_four(uint64_t addr, int dtype, int i, const float (&x)[4]) {
    if (dtype == ASPIS_F32) {
        store_vec<F32, USE>((MutPtr<F32>)addr + i, F32::pack(x));
        return;
    }
    const float y[8] = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    const u32x4 w = dtype == ASPIS_BF16 ? BF16::pack(y) : F16::pack(y);
    u32x2_at2 GLOBAL *q = (u32x2_at2 GLOBAL *)((uint16_t GLOBAL *)addr + i);
    if constexpr (USE == Use::Once) __builtin_nontemporal_store((u32x2_at2){w.x, w.y}, q);
    else *q = (u32x2_at2){w.x, w.y};
}

__device__ __forceinline__ float load_one(uint64_t addr, int dtype, int i) {
    float x = 0.0f;
    with_type(dtype, [&](auto e) { x = decltype(e)::get(((Ptr<decltype(e)>)addr)[i]); });
    return x;
}
__device__ __forceinline__ void store_one(uint64_t addr, int dtype, int i, float x) {
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

// Chunk k of all the update's tensors.
template <typename Rule>
struct UpdateChunk {
    static constexpr int S = Rule::S, W = S > 0 ? S : 1;
    uint64_t p, s[W], g, copy;
    int n, g_type, copy_type;   // copy_type < 0: no copy

    __device__ __forceinline__ UpdateChunk(const UpdateTables &t, int64_t k) {
        const aspis_chunk c = t.grads[k];
        n = c.n;
        g = c.addr;
        g_type = chunk_type(c);
        p = t.params[k].addr;
#pragma unroll
        for (int j = 0; j < W; ++j) s[j] = j < S ? t.state[j][k].addr : 0;
        copy = 0;
        copy_type = -1;
        if (t.copies != nullptr) {
            const aspis_chunk o = t.copies[k];
            copy = o.addr;
            copy_type = chunk_type(o);
        }
    }

    // Four elements on their way.
    struct Four {
        float x[4], q[4], v[W][4];
    };
    __device__ __forceinline__ void load(int i, Four &f) const {
        if (i + 4 > n) return;
        load_four<Use::Once>(g, g_type, i, f.x);
        load_four<Use::Once>(p, ASPIS_F32, i, f.q);
#pragma unroll
        for (int j = 0; j < S; ++j) load_four<Use::Once>(s[j], ASPIS_F32, i, f.v[j]);
    }
    // Updates elements i to i + 3, which f holds; those below n.
    template <Use OUT>
    __device__ __forceinline__ void finish(const Rule &rule, Coef c, int i, Four &f) const {
        if (i + 4 <= n) {
#pragma unroll
            for (int l = 0; l < 4; ++l) {
                float one[W];
#pragma unroll
                for (int j = 0; j < S; ++j) one[j] = f.v[j][l];
                rule(c(f.x[l]), f.q[l], one);
#pragma unroll
                for (int j = 0; j < S; ++j) f.v[j][l] = one[j];
            }
            store_four<OUT>(p, ASPIS_F32, i, f.q);
#pragma unroll
            for (int j = 0; j < S; ++j) store_four<OUT>(s[j], ASPIS_F32, i, f.v[j]);
            if (copy_type >= 0) store_four<OUT>(copy, copy_type, i, f.q);
            return;
        }
        for (; i < n; ++i) {
            float one[W], y = load_one(p, ASPIS_F32, i);
#pragma unroll
            for (int j = 0; j < S; ++j) one[j] = load_one(s[j], ASPIS_F32, i);
            rule(c(load_one(g, g_type, i)), y, one);
            store_one(p, ASPIS_F32, i, y);
#pragma unroll
            for (int j = 0; j < S; ++j) store_one(s[j], ASPIS_F32, i, one[j]);
            if (copy_type >= 0) store_one(copy, copy_type, i, y);
        }
    }
};

// Long lists: one wave and four elements a lane, so that the memory system
// sees each tensor's lines in order, 1 KB at a time.  The sum is joined
// before.  Memory bounds it: AdamW on 871M parameters with bf16 gradients
// and copy moves 24.4 GB in 3.72 to 4.01 ms by where the tensors lie, 6.1 to
// 6.5 TB/s, each byte once.
constexpr int kUpdateBlock = 64;
constexpr int kUpdateParts = kChunk / (4 * kUpdateBlock);

template <typename Rule>
__global__ __launch_bounds__(kUpdateBlock) void
update_kernel(UpdateTables t, int64_t first, int64_t step, NormIn in, Rule rule, bool skip) {
    const double sumsq = *in.sumsq;
    if (blockIdx.x == 0 && threadIdx.x == 0) *in.norm = (float)sqrt(sumsq);
    if (skip && !norm_is_finite(sumsq)) return;
    const UpdateChunk<Rule> c(t, first + step * (blockIdx.x / kUpdateParts));
    const int i = ((int)(blockIdx.x % kUpdateParts) * kUpdateBlock + (int)threadIdx.x) * 4;
    typename UpdateChunk<Rule>::Four f;
    c.load(i, f);
    c.template finish<Use::Once>(rule, coefficient(sumsq, in.max_norm), i, f);
}

// Shorter ones: a chunk per workgroup, on its way while the workgroup joins
// the partial sums; one launch less.  SGD with momentum on 11.2M f32 moves
// 223 MB in 32 to 34 us, 6.6 to 7.0 TB/s, the gradients coming from the cache.
constexpr int kWideBlock = 512;

template <typename Rule>
__global__ __launch_bounds__(kWideBlock) void
wide_update_kernel(UpdateTables t, NormIn in, Rule rule, bool skip) {
    constexpr int N = kChunk / (4 * kWideBlock);
    const UpdateChunk<Rule> c(t, blockIdx.x);
    typename UpdateChunk<Rule>::Four f[N];
#pragma unroll
    for (int u = 0; u < N; ++u) c.load((u * kWideBlock + (int)threadIdx.x) * 4, f[u]);
    const double sumsq = take_sumsq<kWideBlock>(in);
    if (skip && !norm_is_finite(sumsq)) return;
    const Coef coef = coefficient(sumsq, in.max_norm);
#pragma unroll
    for (int u = 0; u < N; ++u)
        c.template finish<Use::Once>(rule, coef, (u * kWideBlock + (int)threadIdx.x) * 4, f[u]);
}

// ---------------------------------------------------------------------------
// short lists: everything in one workgroup and one launch

struct NoApply {
    __device__ void operator()(int64_t, int, double) const {}
};
struct Scale {
    const aspis_chunk *table, *out;
    double max_norm;
    __device__ void operator()(int64_t k, int t, double sumsq) const {
        const Coef coef = coefficient(sumsq, max_norm);
        if (out == nullptr && coef.one()) return;
        const aspis_chunk c = table[k];
        const uint64_t to = out != nullptr ? out[k].addr : c.addr;
        with_type(chunk_type(c), [&](auto e) {
            typedef decltype(e) E;
            Tile<E> tile;
            tile.template load<Use::Again>((Ptr<E>)c.addr, c.n, t);
            tile.template store<Use::Again>((MutPtr<E>)to, c.n, t, coef);
        });
    }
};
template <typename Rule>
struct Update {
    UpdateTables tables;
    Rule rule;
    double max_norm;
    bool skip;
    __device__ void operator()(int64_t k, int t, double sumsq) const {
        if (skip && !norm_is_finite(sumsq)) return;
        const Coef coef = coefficient(sumsq, max_norm);
        const UpdateChunk<Rule> c(tables, k);
        for (int i = t * 4; i < c.n; i += 4 * 256) {
            typename UpdateChunk<Rule>::Four f;
            c.load(i, f);
            c.template finish<Use::Again>(rule, coef, i, f);
        }
    }
};

// Four groups of 256 threads take the chunks in turn: their sums (one per
// wave), the norm (joined as list_sumsq_kernel and block_sum_of join a
// workgroup per chunk), then what is applied to them.  Latency bounds it: of 7,850
// elements in two tensors a norm takes 2.1 us, a clip 3.4, an SGD update 4.6.
constexpr int kSoloBlock = 1024;
static_assert(kSoloChunks == 16, "16 lanes hold the chunks' sums");

template <typename Apply>
__global__ __launch_bounds__(kSoloBlock) void
solo_kernel(const aspis_chunk *__restrict__ table, int n_chunks, const aspis_chunk *tensors,
            int n_tensors, bool have_sumsq, NormIn in, float *each, Apply apply) {
    __shared__ double sums[kSoloChunks * 4];
    const int t = threadIdx.x % 256, group = threadIdx.x / 256;
    double total;
    if (have_sumsq) {
        total = *in.sumsq;
    } else {
        for (int k = group; k < n_chunks; k += kSoloBlock / 256) {
            const double s = lanes_sum<64>(chunk_squares<Use::Again>(table[k], t));
            if (t % 64 == 0) sums[k * 4 + t / 64] = s;
        }
        __syncthreads();
        const int k = threadIdx.x % kSoloChunks;
        const double *of = sums + k * 4;
        total = lanes_sum<kSoloChunks>(k < n_chunks ? of[0] + of[1] + of[2] + of[3] : 0.0);
        if (threadIdx.x == 0) *in.sumsq = total;
        if (each != nullptr)
            for (int i = threadIdx.x; i < n_tensors; i += kSoloBlock) {
                const aspis_chunk c = tensors[i];
                double s = 0.0;
                for (int j = 0; j < c.n * 4; ++j) s += sums[c.addr * 4 + j];
                each[i] = (float)sqrt(s);
            }
    }
    if (threadIdx.x == 0) *in.norm = (float)sqrt(total);
    for (int k = group; k < n_chunks; k += kSoloBlock / 256) apply(k, t, total);
}

// ---------------------------------------------------------------------------
// rows

// A row in the registers of L lanes, R vectors each: read once, its norm,
// written once.  L <= 64: B / L rows per workgroup; L == B: one.  Memory
// bounds it: 6,900 rows of 10,007 f16 in 47.2 us, 5.9 TB/s; few rows are
// latency (15 of 7,850 f32: 3.5 us).
template <typename E, int L, int B, int R>
__global__ __launch_bounds__(B) void row_kernel(RowArgs a) {
    constexpr int G = B / L;
    const int lane = threadIdx.x % L;
    for (int64_t row0 = (int64_t)blockIdx.x * G; row0 < a.rows; row0 += (int64_t)gridDim.x * G) {
        const int64_t row = row0 + threadIdx.x / L;
        const int d = row < a.rows ? (int)a.d : 0;
        Span<E, L, R> span;
        span.template load<Use::Once>((Ptr<E>)a.x + row * a.ld, d, lane);
        double s = span.squares();
        if constexpr (L == B) s = block_sum<B>(s);
        else s = lanes_sum<L>(s);
        if (d > 0 && lane == 0 && a.norms != nullptr) a.norms[row] = (float)sqrt(s);
        if (a.out == nullptr) continue;
        const Coef c = coefficient(s, a.max_norm);
        if (a.out == a.x && c.one()) continue;
        span.template store<Use::Once>((MutPtr<E>)a.out + row * a.ldo, d, lane, c);
    }
}

__global__ __launch_bounds__(kListBlock) void empty_rows_kernel(float *norms, int64_t rows) {
    for (int64_t i = blockIdx.x * (int64_t)kListBlock + threadIdx.x; i < rows;
         i += (int64_t)gridDim.x * kListBlock)
        norms[i] = 0.0f;
}

// A long row is cut into parts, each summed by 256 threads in the same order
// whichever kernel does it, and its parts' sums are added in order: a row's
// norm depends on its elements and length alone.
//
// part_kernel: a part stays in the registers of a workgroup, R vectors a
// thread, which publishes its sum of squares, waits for the row's total and
// writes its part, so the row crosses the memory bus once each way: 91 rows
// of 11.2M f32 in 1.50 ms, 5.4 TB/s (segment_kernel, which reads them twice:
// 2.15 ms).  The device holds two such rows at a time, and a row's workgroups
// load, wait and store together; update_kernel, which waits for nothing, moves
// up to 6.5 TB/s.
//
// A sum is published as one 64-bit word that is never kUnset (a NaN that
// came from f32 or f16 has zeros in its low bits), so a reader needs no
// other flag.  The last workgroup of a row to arrive joins the row's sums,
// in order.  Whether a row's workgroups run together is up to the device:
// the wait for the total is bounded, and a workgroup that gives up lists its
// part for redo_kernel, which reads it again.  The bound changes the time
// alone, never a result.
constexpr uint64_t kUnset = ~uint64_t(0);
constexpr int kLine = 16;            // 8-byte words of a 128-byte line
constexpr int kPartBlock = 256;
constexpr int64_t kPatience = 10000; // ticks of 10 ns

struct PartArgs {
    RowArgs a;
    int32_t parts, length;      // of a row; elements of a part, the last one's fewer
    int64_t patience;
    uint64_t *sums, *totals;    // [rows][parts], [rows] lines; kUnset at the start
    uint32_t *arrived;          // [rows] lines, 0 at the start
    uint32_t *left;             // [0]: the number of parts given up; from [1] on: which
};

__global__ __launch_bounds__(kListBlock) void part_init_kernel(PartArgs g) {
    const int64_t step = (int64_t)gridDim.x * kListBlock;
    for (int64_t i = blockIdx.x * (int64_t)kListBlock + threadIdx.x; i < g.a.rows * g.parts;
         i += step) {
        g.sums[i] = kUnset;
        if (i < g.a.rows) {
            g.totals[i * kLine] = kUnset;
            g.arrived[i * 2 * kLine] = 0;
        }
        if (i == 0) *g.left = 0;
    }
}

__device__ __forceinline__ void publish(uint64_t *at, double v) {
    __hip_atomic_store(at, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t peek(const uint64_t *at) {
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename E, int R, int WAVES>
__global__ __launch_bounds__(kPartBlock, WAVES) void part_kernel(PartArgs g) {
    __shared__ bool last;
    __shared__ uint64_t got;
    const int64_t row = blockIdx.x / (uint32_t)g.parts;
    const int part = (int)(blockIdx.x % (uint32_t)g.parts);
    const int64_t at = (int64_t)part * g.length;
    const int n = (int)(g.a.d - at < g.length ? g.a.d - at : g.length);
    Span<E, kPartBlock, R> span;
    span.template load<Use::Once>((Ptr<E>)g.a.x + row * g.a.ld + at, n, threadIdx.x);
    const double s = block_sum<kPartBlock>(span.squares());
    uint64_t *sums = g.sums + row * g.parts, *its_total = g.totals + row * kLine;
    if (threadIdx.x == 0) {
        publish(sums + part, s);
        last = atomicAdd(g.arrived + row * 2 * kLine, 1u) == (uint32_t)g.parts - 1;
    }
    __syncthreads();
    double total;
    if (last) {   // every sum of the row has been published: no long wait
        double v = 0.0;
        for (int i = threadIdx.x; i < g.parts; i += kPartBlock) {
            uint64_t w;
            do w = peek(sums + i);
            while (w == kUnset);
            v += __builtin_bit_cast(double, w);
        }
        total = block_sum<kPartBlock>(v);
        if (threadIdx.x == 0) {
            publish(its_total, total);
            if (g.a.norms != nullptr) g.a.norms[row] = (float)sqrt(total);
        }
    } else {
        if (threadIdx.x == 0) {
            const int64_t start = wall_clock64();
            uint64_t w = peek(its_total);
            while (w == kUnset && (int64_t)wall_clock64() - start < g.patience) {
                __builtin_amdgcn_s_sleep(1);
                w = peek(its_total);
            }
            if (w == kUnset) g.left[1 + atomicAdd(g.left, 1u)] = blockIdx.x;
            got = w;
        }
        __syncthreads();
        if (got == kUnset) return;
        total = __builtin_bit_cast(double, got);
    }
    const Coef c = coefficient(total, g.a.max_norm);
    if (g.a.out == g.a.x && c.one()) return;
    span.template store<Use::Once>((MutPtr<E>)g.a.out + row * g.a.ldo + at, n, threadIdx.x, c);
}

// The parts that were given up; their rows' totals are all there now.
template <typename E, int R>
__global__ __launch_bounds__(kPartBlock) void redo_kernel(PartArgs g) {
    const uint32_t n_left = *g.left;
    for (uint32_t i = blockIdx.x; i < n_left; i += gridDim.x) {
        const uint32_t item = g.left[1 + i];
        const int64_t row = item / (uint32_t)g.parts;
        const int64_t at = (int64_t)(item % (uint32_t)g.parts) * g.length;
        const int n = (int)(g.a.d - at < g.length ? g.a.d - at : g.length);
        const Coef c =
            coefficient(__builtin_bit_cast(double, g.totals[row * kLine]), g.a.max_norm);
        if (g.a.out == g.a.x && c.one()) continue;
        Span<E, kPartBlock, R> span;
        span.template load<Use::Once>((Ptr<E>)g.a.x + row * g.a.ld + at, n, threadIdx.x);
        span.template store<Use::Once>((MutPtr<E>)g.a.out + row * g.a.ldo + at, n, threadIdx.x, c);
    }
}

// Rows longer than the registers hold, and few short ones (two launches):
// one launch sums the parts of rows [sum0, sum0 + ...) and scales those of the
// rows before, whose sums are there and which the last-level cache still
// holds; the two kinds of workgroups are spread evenly over the launch.  40
// rows of 100,000 f32 (16 MB): 14.5 us, two launches and the cache's rate.
struct SegArgs {
    RowArgs a;
    int32_t parts, length;    // of a row, summed by a workgroup each
    int32_t tiles;            // chunks of a row, scaled by a workgroup each
    int64_t scale0, sum0;
    int64_t n_scale, n_sum;   // workgroups of each kind
};

template <typename E>
__global__ __launch_bounds__(kListBlock) void segment_kernel(SegArgs g) {
    const int64_t b = blockIdx.x, all = g.n_scale + g.n_sum;
    const int64_t before = b * g.n_sum / all;
    if ((b + 1) * g.n_sum / all > before) {
        const int64_t row = g.sum0 + before / g.parts;
        const int part = (int)(before % g.parts);
        int64_t at = (int64_t)part * g.length;
        const int64_t end = at + g.length < g.a.d ? at + g.length : g.a.d;
        const Ptr<E> p = (Ptr<E>)g.a.x + row * g.a.ld;
        double acc[2] = {0.0, 0.0};
        for (; at < end; at += kChunk) {
            Tile<E> tile;
            const int n = (int)(end - at < kChunk ? end - at : kChunk);
            if (g.a.out == nullptr) tile.template load<Use::Once>(p + at, n, threadIdx.x);
            else tile.template load<Use::Again>(p + at, n, threadIdx.x);
            tile.squares(acc);
        }
        const double s = block_sum<kListBlock>(acc[0] + acc[1]);
        if (threadIdx.x == 0) g.a.scratch[row * g.parts + part] = s;
        return;
    }
    const int64_t item = b - before;
    const int64_t row = g.scale0 + item / g.tiles;
    const int64_t at = item % g.tiles * kChunk;
    const int n = (int)(g.a.d - at < kChunk ? g.a.d - at : kChunk);
    const double s = block_sum_of<kListBlock>(g.a.scratch + row * g.parts, g.parts);
    if (at == 0 && threadIdx.x == 0 && g.a.norms != nullptr) g.a.norms[row] = (float)sqrt(s);
    const Coef c = coefficient(s, g.a.max_norm);
    if (g.a.out == g.a.x && c.one()) return;
    Tile<E> tile;
    tile.template load<Use::Once>((Ptr<E>)g.a.x + row * g.a.ld + at, n, threadIdx.x);
    tile.template store<Use::Once>((MutPtr<E>)g.a.out + row * g.a.ldo + at, n, threadIdx.x, c);
}

// The norms alone of long rows, from their segments' sums.
__global__ __launch_bounds__(kListBlock) void segment_norm_kernel(const double *sums, int parts,
                                                                  float *norms) {
    const double s = block_sum_of<kListBlock>(sums + (int64_t)blockIdx.x * parts, parts);
    if (threadIdx.x == 0) norms[blockIdx.x] = (float)sqrt(s);
}

constexpr int64_t kMaxGrid = int64_t(1) << 23;   // workgroups of one launch
// Bytes of rows per launch of segment_kernel: what the last-level cache
// holds until the next launch scales it, next to what that one reads.
constexpr int64_t kGroupBytes = 64 << 20;

template <typename E, int L, int B, int R>
void start_rows(const RowArgs &a, hipStream_t s) {
    const int64_t blocks = (a.rows + B / L - 1) / (B / L);
    const int64_t cap = 1 << 20;
    row_kernel<E, L, B, R><<<(unsigned)(blocks < cap ? blocks : cap), B, 0, s>>>(a);
}

// Workgroups of part_kernel<.., 24, 4> the device runs at once: four a
// compute unit.  Looked up once per device (relaxed atomics: concurrent
// first calls store the same value).
int parts_at_once() {
    static std::atomic<int> known[64];
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
    cus = known[dev].load(std::memory_order_relaxed);
    if (cus == 0) {
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
            return 0;
        known[dev].store(cus, std::memory_order_relaxed);
    }
    return 4 * cus;
}

template <typename E, int R, int WAVES>
hipError_t start_parts(const RowArgs &a, const RowPlan &plan, hipStream_t s) {
    PartArgs g{};
    g.parts = plan.parts;
    g.length = plan.length;
    // a row takes three quarters of the device at most: with less to run on,
    // waiting for its other parts would be in vain
    g.patience = a.wait && 4 * (int64_t)plan.parts <= 3 * (int64_t)parts_at_once() ? kPatience : 0;
    const int64_t step = kMaxGrid / plan.parts;   // rows a launch
    for (int64_t r = 0; r < a.rows; r += step) {
        g.a = a;
        g.a.rows = a.rows - r < step ? a.rows - r : step;
        g.a.x = (const char *)a.x + r * a.ld * (int64_t)sizeof(typename E::T);
        g.a.out = (char *)a.out + r * a.ldo * (int64_t)sizeof(typename E::T);
        g.a.norms = a.norms != nullptr ? a.norms + r : nullptr;
        g.totals = (uint64_t *)a.scratch;
        g.arrived = (uint32_t *)(g.totals + g.a.rows * kLine);
        g.sums = (uint64_t *)(g.arrived + g.a.rows * 2 * kLine);
        g.left = (uint32_t *)(g.sums + g.a.rows * g.parts);
        part_init_kernel<<<64, kListBlock, 0, s>>>(g);
        const unsigned items = (unsigned)(g.a.rows * g.parts);
        part_kernel<E, R, WAVES><<<items, kPartBlock, 0, s>>>(g);
        redo_kernel<E, R><<<items < 512 ? items : 512, kPartBlock, 0, s>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename E>
hipError_t start_segments(const RowArgs &a, const RowPlan &plan, hipStream_t s) {
    SegArgs g{};
    g.a = a;
    g.parts = plan.parts;
    g.length = plan.length;
    g.tiles = (int32_t)chunks_of(a.d);
    const int64_t bytes = a.d * (int64_t)sizeof(typename E::T);
    int64_t step = a.out != nullptr ? kGroupBytes / bytes : kMaxGrid / plan.parts;
    const int64_t most = kMaxGrid / ((int64_t)g.tiles + g.parts);
    if (step > most) step = most;
    if (step < 1) step = 1;
    for (int64_t r = 0; r < a.rows + (a.out != nullptr ? step : 0); r += step) {
        auto group = [&](int64_t first) {   // rows of the group that begins there
            if (first < 0 || first >= a.rows) return (int64_t)0;
            return a.rows - first < step ? a.rows - first : step;
        };
        g.sum0 = r;
        g.scale0 = r - step;
        g.n_sum = group(r) * g.parts;
        g.n_scale = a.out != nullptr ? group(r - step) * g.tiles : 0;
        segment_kernel<E><<<(unsigned)(g.n_sum + g.n_scale), kListBlock, 0, s>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.out == nullptr)
        for (int64_t r = 0; r < a.rows; r += kMaxGrid) {
            const int64_t n = a.rows - r < kMaxGrid ? a.rows - r : kMaxGrid;
            segment_norm_kernel<<<(unsigned)n, kListBlock, 0, s>>>(a.scratch + r * plan.parts,
                                                                   plan.parts, a.norms + r);
        }
    return hipGetLastError();
}

template <typename E>
hipError_t rows_of(const RowArgs &a, hipStream_t s) {
    const RowPlan plan = row_plan(a.rows, a.d, (int)sizeof(typename E::T));
    if (plan.kind == RowKind::Parts && a.out != nullptr)
        return plan.vecs == 8 ? start_parts<E, 8, 6>(a, plan, s) : start_parts<E, 24, 4>(a, plan, s);
    if (plan.kind != RowKind::Registers) return start_segments<E>(a, plan, s);
    const int64_t nv = (a.d + E::V - 1) / E::V;
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

// Chunks at the end of a list that the last-level cache (256 MB) keeps from
// one pass to the next, of f32.  Of 180 MB clipped: 85.7 us, with 192 MB
// kept 87.6, with 320 MB 86.2.
constexpr int64_t kKeepChunks = (int64_t)256 * 1024 * 1024 / (4 * kChunk);
// From here on the partial sums are joined by a launch of their own; below,
// by every workgroup that scales a chunk.  Joined apart and by every workgroup,
// us: a clip of 3,500 chunks 27.4 and 26.2, of 8,000 60.6 both ways; SGD of 5,000
// 75.7 and 75.4, of 9,000 131 and 133, of 16,000 226 and 237.
constexpr int64_t kJoinChunks = 8192;

// Chunks of one launch that takes them all: its threads stay below 2^32.
constexpr int64_t kLaunchChunks = int64_t(1) << 21;

// Calls launch(first chunk, step, chunks) over a list: forwards, or the last
// chunk first where the list is longer than what the cache keeps of it.
template <typename F>
hipError_t over_chunks(int64_t n_chunks, F &&launch) {
    const bool backwards = n_chunks > kKeepChunks;
    for (int64_t done = 0; done < n_chunks; done += kLaunchChunks) {
        const int64_t n = n_chunks - done < kLaunchChunks ? n_chunks - done : kLaunchChunks;
        launch(backwards ? n_chunks - 1 - done : done, backwards ? int64_t(-1) : int64_t(1),
               (unsigned)n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename Apply>
hipError_t start_solo(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors,
                      bool have_sumsq, const NormIn &in, float *each, const Apply &apply,
                      hipStream_t s) {
    solo_kernel<<<1, kSoloBlock, 0, s>>>(table, (int)n_chunks, table + n_chunks, n_tensors,
                                         have_sumsq, in, each, apply);
    return hipGetLastError();
}

// The norm pass and, when asked, its joining; afterwards in says where the
// sum is.
hipError_t start_sumsq(const aspis_chunk *table, int64_t n_chunks, double *ws, bool read_again,
                       bool join, int32_t n_tensors, float *each, NormIn *in, hipStream_t s) {
    const int groups = (int)(n_chunks < kNormGroups ? n_chunks : kNormGroups);
    const int group = (int)(n_chunks / (4 * kNormGroups) < 1    ? 1
                            : n_chunks / (4 * kNormGroups) > 16 ? 16
                                                                : n_chunks / (4 * kNormGroups));
    const int64_t keep = !read_again ? n_chunks : n_chunks > kKeepChunks ? n_chunks - kKeepChunks : 0;
    double *runs = each != nullptr ? ws + kNormGroups : nullptr;
    list_sumsq_kernel<<<groups, kListBlock, 0, s>>>(table, n_chunks, group, keep, ws, runs);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    in->partial = ws;
    in->n_partial = groups;
    if (!join) return hipSuccess;
    list_norm_kernel<<<each != nullptr ? 1u + (unsigned)n_tensors : 1u, kListBlock, 0, s>>>(
        table + n_chunks, group, *in, runs, each);
    in->n_partial = 0;
    return hipGetLastError();
}

template <typename Rule>
hipError_t update_list(const UpdateTables &t, int64_t n_chunks, bool have_sumsq, double *ws,
                       NormIn in, const Rule &rule, bool skip, hipStream_t s) {
    if (n_chunks <= kSoloUpdate)
        return start_solo(t.grads, n_chunks, 0, have_sumsq, in, nullptr,
                          Update<Rule>{t, rule, in.max_norm, skip}, s);
    // AdamW's seven streams gain from update_kernel's order earlier: joined
    // apart and by every workgroup, 2,000 chunks take 45.9 and 42.5 us, 2,700
    // 59.7 and 60.6, 3,500 72.6 and 74.4, 8,000 154 and 161
    const bool join = n_chunks >= (Rule::S > 1 ? kJoinChunks / 3 : kJoinChunks);
    if (!have_sumsq) {
        const hipError_t e = start_sumsq(t.grads, n_chunks, ws, true, join, 0, nullptr, &in, s);
        if (e != hipSuccess) return e;
    }
    if (!join) {
        wide_update_kernel<<<(unsigned)n_chunks, kWideBlock, 0, s>>>(t, in, rule, skip);
        return hipGetLastError();
    }
    return over_chunks(n_chunks, [&](int64_t first, int64_t step, unsigned n) {
        update_kernel<<<n * kUpdateParts, kUpdateBlock, 0, s>>>(t, first, step, in, rule, skip);
    });
}

}  // namespace

hipError_t launch_norm(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors, double *ws,
                       NormIn in, float *each, hipStream_t s) {
    if (n_chunks <= kSoloChunks)
        return start_solo(table, n_chunks, n_tensors, false, in, each, NoApply{}, s);
    return start_sumsq(table, n_chunks, ws, false, true, n_tensors, each, &in, s);
}

hipError_t launch_clip(const aspis_chunk *table, const aspis_chunk *out, int64_t n_chunks,
                       bool have_sumsq, double *ws, NormIn in, hipStream_t s) {
    if (n_chunks <= kSoloClip)
        return start_solo(table, n_chunks, 0, have_sumsq, in, nullptr,
                          Scale{table, out, in.max_norm}, s);
    if (!have_sumsq) {
        const hipError_t e = start_sumsq(table, n_chunks, ws, true, n_chunks >= kJoinChunks, 0,
                                         nullptr, &in, s);
        if (e != hipSuccess) return e;
    }
    return over_chunks(n_chunks, [&](int64_t first, int64_t step, unsigned n) {
        list_scale_kernel<<<n, kListBlock, 0, s>>>(table, out, first, step, in);
    });
}

hipError_t launch_sgd(const aspis_chunk *params, const aspis_chunk *grads,
                      const aspis_chunk *mean, const aspis_chunk *copies, int64_t n_chunks,
                      bool have_sumsq, double *ws, const NormIn &in, const SgdArgs &a, bool skip,
                      hipStream_t s) {
    const UpdateTables t{params, grads, {mean, nullptr}, copies};
    if (mean != nullptr) return update_list(t, n_chunks, have_sumsq, ws, in, Sgd{a}, skip, s);
    return update_list(t, n_chunks, have_sumsq, ws, in, PlainSgd{a}, skip, s);
}

hipError_t launch_adamw(const aspis_chunk *params, const aspis_chunk *grads,
                        const aspis_chunk *mean, const aspis_chunk *square,
                        const aspis_chunk *copies, int64_t n_chunks, bool have_sumsq, double *ws,
                        const NormIn &in, const AdamArgs &a, bool skip, hipStream_t s) {
    return update_list(UpdateTables{params, grads, {mean, square}, copies}, n_chunks, have_sumsq,
                       ws, in, AdamW{a}, skip, s);
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
