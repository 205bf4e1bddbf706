// aspis_policy.hip -- gfx950 kernels of the log-probabilities of tokens and
// of the clipped policy loss with its gradient by the logits.
//
// With z a row of logits, M its maximum, c = log2(e) / temperature and
// S = sum of 2^((z_v - M) c): log p(t) = (z_t - M) / temperature - ln S, and
// the gradient's softmax is 2^((z_v - M) c) / S.
//
// A row's whole vectors are cut into units of 64 lanes and at most 8 vectors a
// lane, by its length and type alone (the elements after the last vector go
// to the first unit, one a lane): each has its own maximum and sum (a lane's
// powers in order, then the lanes), and the units are joined in order.  So a
// row has the same bits whichever kernel takes it and whatever other rows
// the call has: files batched together or one by one give the same gradient.
#include "aspis_tokens.h"

#include <cmath>

#include "aspis_elements.h"

namespace aspis {

namespace {

constexpr int64_t kMaxGrid = int64_t(1) << 22;   // workgroups of one launch

// 2^((z - m) c) as 2^(z c - k), k = m c rounded: one operation and one
// rounding less.  k's rounding is a factor that all powers of a unit share, so
// it cancels where they are divided by their sum; but it is half a step of k,
// which has to be small beside 127: at |k| = 2^20 it is 2^-5, and from 2^31 on the
// largest power itself may be infinite or 0.  Beyond (logits masked by a
// constant, a low temperature) the difference comes first: its operands cannot be
// infinities of both signs.
struct Fast {
    float c, k;
    __device__ float operator()(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, c, -k)); }
};
struct Slow {
    float c, m;   // of -inf alone, which count nothing: differences from 0
    __device__ Slow(float c, float top) : c(c), m(top == -INFINITY ? 0.0f : top) {}
    __device__ float operator()(float z) const { return __builtin_amdgcn_exp2f((z - m) * c); }
};
__device__ __forceinline__ bool is_fast(float m, float c) { return fabsf(m * c) <= 0x1p20f; }

// The factor of a sum of powers relative to `from` that makes it relative to
// `to`, which is not below; each is Fast's k or Slow's m, by its size.
__device__ __forceinline__ float rescale(float from, float to, float c) {
    const float k = from * c;
    const bool fast = is_fast(from, c);
    if (is_fast(to, c)) return __builtin_amdgcn_exp2f(fast ? k - to * c : fmaf(from, c, -(to * c)));
    return fast ? __builtin_amdgcn_exp2f(fmaf(-to, c, k)) : Slow(c, to)(from);
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// A maximum and the sum of the powers relative to it; of -inf alone the sum
// is 0.
struct Stats {
    float m, s;
};

// The same of every lane's, joined in lane order.
__device__ __forceinline__ Stats join_lanes(Stats p, float c) {
    const float m = lanes_join<64>(p.m, Max());
    return {m, lanes_join<64>(p.s == 0.0f ? 0.0f : p.s * rescale(p.m, m, c), Sum())};
}

// Of N vectors a lane, and one element.  Any power near the largest will do
// as the scale, since a sum of up to kRoom relative to it loses nothing in
// f32: the largest of one element in V, which takes a third of the time of
// the largest of all, and that one only where the sum says so.
constexpr float kRoom = 0x1p60f;

template <typename E, int N>
__device__ __forceinline__ Stats unit_stats(const u32x4 *v, float tail, float c) {
    auto sum = [&](float m) {
        float s = 0.0f;
        auto add = [&](auto power) {
#pragma unroll
            for (int r = 0; r < N; ++r) {
                u32x4 again = v[r];
                asm volatile("" : "+v"(again));   // unpacked anew: kept, it takes twice the registers
                float x[E::V];
                E::unpack(again, x);
#pragma unroll
                for (int j = 0; j < E::V; ++j) s += power(x[j]);
            }
            s += power(tail);
        };
        if (__builtin_amdgcn_readfirstlane(is_fast(m, c))) add(Fast{c, m * c});
        else add(Slow(c, m));
        return lanes_join<64>(s, Sum());
    };
    float m = tail;
#pragma unroll
    for (int r = 0; r < N; ++r) {
        float x[E::V];
        E::unpack(v[r], x);
        m = fmaxf(m, x[0]);
    }
    m = lanes_join<64>(m, Max());
    float s = sum(m);
    if (__builtin_amdgcn_readfirstlane(m == -INFINITY || !(s <= kRoom))) {
        m = tail;
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float x[E::V];
            E::unpack(v[r], x);
#pragma unroll
            for (int j = 0; j < E::V; ++j) m = fmaxf(m, x[j]);
        }
        m = lanes_join<64>(m, Max());
        s = sum(m);
    }
    return {m, s};
}

// e^x - 1 - x: by its series near 0, where the difference would cancel.
__device__ __forceinline__ float exp_rest(float x) {
    if (!(fabsf(x) <= 0.5f)) return expf(x) - 1.0f - x;
    float p = 1.0f;
#pragma unroll
    for (int k = 10; k >= 3; --k) p = fmaf(p * x, 1.0f / (float)k, 1.0f);
    return 0.5f * x * x * p;
}

// What a position adds to the sums, and the factor of its gradient.
struct Terms {
    float loss, kl, cut, coef;
};
__device__ __forceinline__ Terms terms_of(const PolicyArgs &a, int64_t row, float weight, float lp) {
    const float adv = a.advantage[row], ratio = expf(lp - a.old[row]);
    const bool cut = adv > 0.0f ? ratio > a.clip_high : adv < 0.0f && ratio < a.clip_low;
    // (no advantage, no gain: not even of an infinite ratio)
    const float gain = adv == 0.0f ? 0.0f
                       : cut       ? (adv > 0.0f ? a.clip_high : a.clip_low) * adv
                                   : ratio * adv;
    Terms t{-gain, 0.0f, cut ? 1.0f : 0.0f, cut ? 0.0f : -gain};
    if (a.ref != nullptr) {
        const float x = a.ref[row] - lp;
        t.kl = exp_rest(x);
        if (a.kl != 0.0f) {
            t.loss += a.kl * t.kl;
            t.coef -= a.kl * (t.kl + x);   // 1 - e^x
        }
    }
    t.coef = weight * t.coef * a.grad_scale;
    return t;
}

// The position's token, or -1 where it is left out; its weight.  (A row is a
// wave's at least: the same in all lanes.)
__device__ __forceinline__ int take_token(const PolicyArgs &a, int64_t row, float &weight) {
    weight = a.sums != nullptr ? a.weight[row] : 1.0f;
    return __builtin_amdgcn_readfirstlane(weight == 0.0f ? -1 : a.tokens.get(row, a.vocab));
}

struct Scratch {
    double *terms;   // [3][rows]
    double *partial; // [3][sum_groups]
    Stats *stats;    // [rows][units]
    float *at;       // [rows]: the token's logit
};

// Writes down what a position adds to the sums, and its log-probability.
__device__ __forceinline__ void put_row(const PolicyArgs &a, const Scratch &w, int64_t row,
                                        bool used, float weight, float lp, const Terms &t) {
    a.logps[row] = lp;
    if (a.sums == nullptr) return;
    w.terms[row] = used ? (double)weight * t.loss : 0.0;
    w.terms[a.rows + row] = used ? (double)weight * t.kl : 0.0;
    w.terms[2 * a.rows + row] = used ? (double)weight * t.cut : 0.0;
}

// Element i of a row, fewer than 2^30 bytes on: the row's address stays in
// scalar registers.
template <typename P>
__device__ __forceinline__ P element(P row, int i) {
    typedef const char GLOBAL *Bytes;
    return (P)((Bytes)row + (uint32_t)i * (uint32_t)sizeof(*row));
}

// The whole vectors lane, lane + step, ... of a row of nv; -inf past them.
// 16-bit rows that begin in the middle of a word are loaded from one element
// earlier, in the same word, and shifted (align) once they are there: 8,192
// rows of 128,003 bf16, half of them such, took 810 us so and 902 without.
// (Stores shifted alike took longer, 4,096 rows 471 instead of 438 us; so did
// whole 16-byte blocks read and written, by shifts of 0 to 7 elements.)
template <typename E, int N>
struct Logits {
    static_assert(N <= 16, "a lane each");
    u32x4 v[N];
    uint32_t past;   // lane r's: the element after the last lane's vector r, but one
    uint32_t end;    // the last element of the row's last vector
    __device__ __forceinline__ static bool odd(Ptr<E> row) {
        return E::V == 8 && __builtin_amdgcn_readfirstlane((int)((uint64_t)row & 2)) != 0;
    }
    __device__ __forceinline__ void load(Ptr<E> row, int lane, int step, int nv) {
        const bool shift = odd(row);
        const Ptr<E> from = shift ? row - 1 : row;
#pragma unroll
        for (int r = 0; r < N; ++r) {
            v[r] = (u32x4){E::kLowest, E::kLowest, E::kLowest, E::kLowest};
            if (lane < nv - r * step)
                v[r] = load_vec<E, Use::Once>(element(from + r * step * E::V, lane * E::V));
        }
        if (E::V != 8 || !shift) return;
        const int l = threadIdx.x % 64, i = lane - l + 63 + l * step;
        past = end = E::kLowest;
        if (l < N && i < nv) past = *(const uint16_t GLOBAL *)(row + i * E::V + 7);
        if (nv > 0) end = *(const uint16_t GLOBAL *)(row + nv * E::V - 1);
    }
    // Vectors FROM to FROM + M - 1 into their places.
    template <int FROM, int M>
    __device__ __forceinline__ void align(Ptr<E> row, int lane, int step, int nv) {
        if (E::V != 8 || !odd(row)) return;
        const int first = __builtin_amdgcn_readfirstlane(lane);
#pragma unroll
        for (int r = FROM; r < FROM + M; ++r) {
            const u32x4 a = v[r];
            uint32_t next = __builtin_amdgcn_update_dpp(0, (int)a.x, 0x130, 0xF, 0xF, true);
            const uint32_t last = __builtin_amdgcn_readlane(past, r);
            next = threadIdx.x % 64 == 63 ? last : next;
            const int i = first + r * step;
            if (i < nv && nv <= i + 64 && lane + r * step == nv - 1) next = end;
            v[r] = (u32x4){__builtin_amdgcn_alignbit(a.y, a.x, 16),
                           __builtin_amdgcn_alignbit(a.z, a.y, 16),
                           __builtin_amdgcn_alignbit(a.w, a.z, 16), next << 16 | a.w >> 16};
        }
    }
};

// What a row's gradient is made of.
struct Grad {
    float m, c, by, own;   // -(the factor) / S; the token's own element
};

// The gradient of a vector's logits.
template <typename E>
__device__ __forceinline__ u32x4 make_grad(u32x4 v, const Grad &g) {
    asm volatile("" : "+v"(v));
    float x[E::V];
    E::unpack(v, x);
    if (__builtin_amdgcn_readfirstlane(is_fast(g.m, g.c))) {
        const Fast power{g.c, g.m * g.c};
#pragma unroll
        for (int j = 0; j < E::V; ++j) x[j] = power(x[j]) * g.by;
    } else {
        const Slow power(g.c, g.m);
#pragma unroll
        for (int j = 0; j < E::V; ++j) x[j] = power(x[j]) * g.by;
    }
    return E::pack(x);
}
// The gradient of the vectors in their place.
template <typename E, int N>
__device__ __forceinline__ void store_grad(MutPtr<E> out, int lane, int step, int nv, const u32x4 *v,
                                           const Grad &g) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const u32x4 w = make_grad<E>(v[r], g);
        if (lane < nv - r * step) store_vec<E, Use::Once>(element(out + r * step * E::V, lane * E::V), w);
    }
}
// ... and of an element after them, `tail`, in the first lanes.
template <typename E>
__device__ __forceinline__ void store_tail(MutPtr<E> out, int lane, int first, int n, float tail,
                                           const Grad &g) {
    if (first + lane >= n) return;
    const float p = is_fast(g.m, g.c) ? Fast{g.c, g.m * g.c}(tail) : Slow(g.c, g.m)(tail);
    out[first + lane] = put_product<E>(p * g.by);
}

// The end of a row's statistics: its log-probability, terms and gradient.
__device__ __forceinline__ Grad finish_row(const PolicyArgs &a, const Scratch &w, int64_t row,
                                           float weight, float z, Stats st, float c, bool writes) {
    // (log2 of the power of the token, in f64: one rounding, in lp; f32 may not hold the difference)
    const double x = is_fast(st.m, c) ? ((double)z * c - (double)(st.m * c)) * 0.6931471805599453
                                      : ((double)z - (double)st.m) * a.inv_temperature;
    const float p = (is_fast(st.m, c) ? Fast{c, st.m * c}(z) : Slow(c, st.m)(z)) / st.s;
    // ln S from its exponent and mantissa: S may lie far above 1, where an f32
    // logarithm of all of it would lose what x cancels
    const double ln_s = (double)logf(__builtin_amdgcn_frexp_mantf(st.s)) +
                        0.6931471805599453 * __builtin_amdgcn_frexp_expf(st.s);
    float lp = (float)(x - ln_s);
    // where the others' share is below f32's, and where a rounding went past 1
    if (p >= 1.0f || lp > 0.0f) lp = 0.0f;
    Terms t{0.0f, 0.0f, 0.0f, 0.0f};
    if (a.sums != nullptr) t = terms_of(a, row, weight, lp);
    if (writes) put_row(a, w, row, true, weight, lp, t);
    return {st.m, c, -t.coef / st.s, t.coef * (1.0f - p)};
}

template <typename E>
__device__ __forceinline__ void zero_row(MutPtr<E> out, int64_t first, int64_t step, int64_t n) {
    for (int64_t i = first; i < n / E::V; i += step)
        store_vec<E, Use::Once>(out + i * E::V, (u32x4){0, 0, 0, 0});
    for (int64_t i = n / E::V * E::V + first; i < n; i += step) out[i] = E::put(0.0f);
}

// How a row of `vecs` vectors is cut (policy_cut): L lanes hold R vectors each,
// lane l the vectors l, l + L, ...; a wave's are a unit, or, of more than 8,
// its first half is one and its second half another.  Rows of more than
// kBlockVecs vectors: blocks of so many, cut alike.
constexpr int unit_vecs(int r) { return r <= 8 ? r : r / 2; }

// A row in the registers of L lanes: read once, its gradient written once.
// Memory bounds it, and what a workgroup of 1,024 lanes computes while its
// compute unit has no other to load: 8,192 rows of 128,000 bf16 in 767 us, 5.5
// TB/s; of 128,003, a quarter of them left out, in 797, 4.6 TB/s, since a
// wave's stores then begin and end within lines.  A loop over rows that sends
// for the next one's logits while it stores took as long (768, 791).
template <typename E, int L, int R, bool GRAD>
__global__ __launch_bounds__(L < 256 ? 256 : L) void
row_kernel(PolicyArgs a, Scratch w, float c, int64_t first) {
    constexpr int B = L < 256 ? 256 : L, N = unit_vecs(R);
    constexpr int UNITS = L / 64 * (R / N);
    static_assert(UNITS <= 64 && R / N <= 2, "a lane each");
    const int lane = threadIdx.x % L;
    const int64_t row = first + (int64_t)blockIdx.x * (B / L) +
                        __builtin_amdgcn_readfirstlane(threadIdx.x / L);
    if (L < B && row >= a.rows) return;
    float weight;
    const int token = take_token(a, row, weight);
    const MutPtr<E> out = (MutPtr<E>)a.grad + row * a.ldg;
    const int n = (int)a.vocab, nv = n / E::V;
    if (token < 0) {
        if (lane == 0) put_row(a, w, row, false, 0.0f, 0.0f, {});
        if constexpr (GRAD) zero_row<E>(out, lane, L, n);
        return;
    }
    const Ptr<E> z = (Ptr<E>)a.logits + row * a.ld;
    Logits<E, R> x;
    x.load(z, lane, L, nv);
    const float tail = nv * E::V + lane < n ? E::get(z[nv * E::V + lane]) : -INFINITY;
    const float at = E::get(z[token]);
    Stats st;
    if constexpr (UNITS == 1) {
        x.template align<0, N>(z, lane, L, nv);
        st = unit_stats<E, N>(x.v, tail, c);
    } else {
        __shared__ Stats units[UNITS];
        auto unit = [&](auto at) {
            constexpr int U = decltype(at)::value;
            x.template align<U * N, N>(z, lane, L, nv);
            const Stats p = unit_stats<E, N>(x.v + U * N, U == 0 ? tail : -INFINITY, c);
            if (threadIdx.x % 64 == 0) units[U * (L / 64) + threadIdx.x / 64] = p;
        };
        unit(Int<0>());
        if constexpr (R / N > 1) unit(Int<1>());
        __syncthreads();
        const int i = threadIdx.x % 64;
        st = join_lanes(i < UNITS ? units[i] : Stats{-INFINITY, 0.0f}, c);
    }
    const Grad g = finish_row(a, w, row, weight, at, st, c, lane == 0);
    if constexpr (!GRAD) return;
    store_grad<E, R>(out, lane, L, nv, x.v, g);
    store_tail<E>(out, lane, nv * E::V, n, tail, g);
    // the token's own, over what the same lane has just written
    if (lane == (token < nv * E::V ? token / E::V % L : token - nv * E::V)) out[token] = put_product<E>(g.own);
}

// Few rows, and rows longer than the registers of a workgroup: a wave for
// every unit, then one for every unit of the gradient.  Many long rows are read
// twice from memory: 4,096 of 128,003 f32 in 1,282 us (log-probabilities 361), 2.0
// of what a read and a write would take.
template <typename E, int L, int R>
__global__ __launch_bounds__(64) void unit_stats_kernel(PolicyArgs a, Scratch w, float c, int units,
                                                        int64_t first) {
    constexpr int N = unit_vecs(R), OF_BLOCK = L / 64 * (R / N);
    const int64_t item = first + blockIdx.x;
    const int64_t row = item / units;
    const int unit = (int)(item % units), block = unit / OF_BLOCK, of = unit % OF_BLOCK;
    float weight;
    const int token = take_token(a, row, weight);
    if (token < 0) return;
    const Ptr<E> z = (Ptr<E>)a.logits + row * a.ld;
    const int n = (int)a.vocab, nv = n / E::V;
    const int i0 = block * kBlockVecs + of / (L / 64) * N * L + of % (L / 64) * 64 + threadIdx.x;
    Logits<E, N> x;
    x.load(z, i0, L, nv);
    x.template align<0, N>(z, i0, L, nv);
    const int last = nv * E::V + threadIdx.x;
    const float tail = unit == 0 && last < n ? E::get(z[last]) : -INFINITY;
    if (unit == 0 && threadIdx.x == 0) w.at[row] = E::get(z[token]);
    const Stats st = unit_stats<E, N>(x.v, tail, c);
    if (threadIdx.x == 0) w.stats[item] = st;
}

template <typename E, int L, int R>
__global__ __launch_bounds__(64) void unit_grad_kernel(PolicyArgs a, Scratch w, float c, int units,
                                                       int grads, int64_t first) {
    constexpr int N = unit_vecs(R), OF_BLOCK = L / 64 * (R / N);
    const int64_t item = first + blockIdx.x;   // (row, one of the `grads` units written)
    const int64_t row = item / grads;
    const int unit = (int)(item % grads), block = unit / OF_BLOCK, of = unit % OF_BLOCK;
    float weight;
    const int token = take_token(a, row, weight);
    const MutPtr<E> out = (MutPtr<E>)a.grad + row * a.ldg;
    if (token < 0) {
        if (unit == 0 && threadIdx.x == 0) put_row(a, w, row, false, 0.0f, 0.0f, {});
        if (a.grad != nullptr) zero_row<E>(out, unit * 64 + threadIdx.x, grads * 64, a.vocab);
        return;
    }
    Stats p{-INFINITY, 0.0f};
    const Stats *of_row = w.stats + row * units;
    if (units <= 64) {
        if ((int)threadIdx.x < units) p = of_row[threadIdx.x];
    } else {
        // a lane's units first: 64 apart, in order, relative to their maximum
        for (int i = threadIdx.x; i < units; i += 64) p.m = fmaxf(p.m, of_row[i].m);
        for (int i = threadIdx.x; i < units; i += 64) {
            const Stats q = of_row[i];
            p.s += q.s == 0.0f ? 0.0f : q.s * rescale(q.m, p.m, c);
        }
    }
    const Grad g = finish_row(a, w, row, weight, w.at[row], join_lanes(p, c), c,
                              unit == 0 && threadIdx.x == 0);
    if (a.grad == nullptr) return;
    const Ptr<E> z = (Ptr<E>)a.logits + row * a.ld;
    const int n = (int)a.vocab, nv = n / E::V, lane = threadIdx.x;
    const int i0 = block * kBlockVecs + of / (L / 64) * N * L + of % (L / 64) * 64 + lane;
    Logits<E, N> x;
    x.load(z, i0, L, nv);
    x.template align<0, N>(z, i0, L, nv);
    store_grad<E, N>(out, i0, L, nv, x.v, g);
    // the token's own, over what the same lane has just written
    const int of_token = token / E::V - i0;
    if (token < nv * E::V && of_token >= 0 && of_token < N * L && of_token % L == 0)
        out[token] = put_product<E>(g.own);
    if (unit != 0) return;
    if (nv * E::V + lane < n) store_tail<E>(out, lane, nv * E::V, n, E::get(z[nv * E::V + lane]), g);
    if (lane == token - nv * E::V) out[token] = put_product<E>(g.own);
}

// The loss and the two other sums, in fp64 and an order that the number of
// rows fixes: of n terms each, `step` a workgroup; to `to` [3][workgroups],
// or to sums from one workgroup.  Latency bounds it: 2.7 us for a few rows, 5.4
// for 8,192, after rows that take 814.
__global__ __launch_bounds__(1024) void sum_terms_kernel(const double *terms, int64_t n,
                                                         int64_t step, double *to, float *sums) {
    const int64_t from = blockIdx.x * step, end = from + step < n ? from + step : n;
    double s[3] = {0.0, 0.0, 0.0};
    for (int64_t i = from + threadIdx.x; i < end; i += 1024)
#pragma unroll
        for (int k = 0; k < 3; ++k) s[k] += terms[k * n + i];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        s[k] = block_sum<1024>(s[k]);
        if (threadIdx.x != 0) continue;
        if (gridDim.x > 1) to[k * gridDim.x + blockIdx.x] = s[k];
        else sums[k] = (float)s[k];
    }
}

hipError_t start_sums(const PolicyArgs &a, const Scratch &w, hipStream_t s) {
    const unsigned groups = (unsigned)sum_groups(a.rows);
    const int64_t step = (a.rows + groups - 1) / groups;
    sum_terms_kernel<<<groups, 1024, 0, s>>>(w.terms, a.rows, step, w.partial, a.sums);
    if (groups > 1)
        sum_terms_kernel<<<1, 1024, 0, s>>>(w.partial, groups, groups, nullptr, a.sums);
    return hipGetLastError();
}

// Calls launch(first, n) until `blocks` workgroups are launched.
template <typename F>
hipError_t over_blocks(int64_t blocks, F &&launch) {
    for (int64_t first = 0; first < blocks; first += kMaxGrid) {
        launch(first, (unsigned)(blocks - first < kMaxGrid ? blocks - first : kMaxGrid));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Fewer rows than this of 1,024 lanes go by units, as rows longer than a
// workgroup holds do: by units and by rows, 16 rows of 128,003 bf16 14.7 and
// 22.9 us, 64 19.0 and 23.7 (log-probabilities 9.0 and 11.7); 16 of 60,003, of
// 512 lanes, 14.4 and 16.4, but their log-probabilities 8.6 and 7.4.
constexpr int64_t kFewRows = 128;

template <typename E, int L, int R>
hipError_t start_rows(const PolicyArgs &a, const Scratch &w, float c, int units, bool by_units,
                      hipStream_t s) {
    constexpr int B = L < 256 ? 256 : L;
    if (!by_units)
        return over_blocks((a.rows + B / L - 1) / (B / L), [&](int64_t first, unsigned n) {
            first *= B / L;
            if (a.grad != nullptr) row_kernel<E, L, R, true><<<n, B, 0, s>>>(a, w, c, first);
            else row_kernel<E, L, R, false><<<n, B, 0, s>>>(a, w, c, first);
        });
    const hipError_t e = over_blocks(a.rows * units, [&](int64_t first, unsigned n) {
        unit_stats_kernel<E, L, R><<<n, 64, 0, s>>>(a, w, c, units, first);
    });
    if (e != hipSuccess) return e;
    const int grads = a.grad != nullptr ? units : 1;
    return over_blocks(a.rows * grads, [&](int64_t first, unsigned n) {
        unit_grad_kernel<E, L, R><<<n, 64, 0, s>>>(a, w, c, units, grads, first);
    });
}

template <typename E>
hipError_t start_policy(const PolicyArgs &a, hipStream_t s) {
    const PolicyPlan plan = policy_plan(a.rows, a.vocab, sizeof(typename E::T));
    char *const ws = (char *)a.ws;
    const Scratch w{(double *)(ws + plan.terms), (double *)(ws + plan.partial), (Stats *)(ws + plan.stats),
                    (float *)(ws + plan.at)};
    const float c = (float)(1.4426950408889634 * a.inv_temperature);
    const int64_t nv = (a.vocab + E::V - 1) / E::V;
    const PolicyCut cut = policy_cut(nv);
    const bool few = cut.lanes == 1024 && a.rows < kFewRows;
    hipError_t e = hipErrorInvalidValue;
    auto rows = [&](auto lanes, auto vecs) {
        constexpr int L = decltype(lanes)::value, R = decltype(vecs)::value;
        if (cut.lanes == L && cut.vecs == R)
            e = start_rows<E, L, R>(a, w, c, plan.units, few || nv > kBlockVecs, s);
    };
    rows(Int<64>(), Int<1>());
    rows(Int<64>(), Int<2>());
    rows(Int<64>(), Int<4>());
    rows(Int<64>(), Int<8>());
    rows(Int<256>(), Int<4>());
    rows(Int<256>(), Int<6>());
    rows(Int<256>(), Int<8>());
    rows(Int<256>(), Int<10>());
    rows(Int<256>(), Int<16>());
    rows(Int<512>(), Int<10>());
    rows(Int<512>(), Int<16>());
    rows(Int<1024>(), Int<10>());
    rows(Int<1024>(), Int<12>());
    rows(Int<1024>(), Int<16>());
    if (e != hipSuccess || a.sums == nullptr) return e;
    return start_sums(a, w, s);
}

}  // namespace

hipError_t launch_policy(const PolicyArgs &a, hipStream_t s) {
    if (a.dtype == ASPIS_F32) return start_policy<F32>(a, s);
    if (a.dtype == ASPIS_BF16) return start_policy<BF16>(a, s);
    return start_policy<F16>(a, s);
}

}  // namespace aspis
