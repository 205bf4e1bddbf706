// aspis_policy.hip -- gfx950 kernels of the log-probabilities of tokens and
// of the clipped policy loss with its gradient by the logits.
//
// With z a row of logits, M its maximum, c = log2(e) / temperature and
// S = sum of 2^((z_v - M) c): log p(t) = (z_t - M) / temperature - ln S, and
// the gradient's softmax is 2^((z_v - M) c) / S.  The difference z_v - M is
// formed before the product, so that logits at the type's lowest value (a
// mask) cannot turn into infinities of both signs; S and its parts are f32,
// at least 1, and joined in a fixed order.
#include "aspis_tokens.h"

#include <cfloat>
#include <cmath>

#include "aspis_elements.h"

namespace aspis {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kMaxGrid = int64_t(1) << 22;   // workgroups of one launch

// A maximum M and the sum of 2^((z - M) c) over some logits; of none, or of
// -inf alone, M = -inf and S = 0.
struct Stats {
    float m, s;
};
__device__ __forceinline__ float power(float z, float m, float c) {
    return __builtin_amdgcn_exp2f((z - m) * c);
}
// What a part's sum counts in one of maximum m (its own maximum at least).
__device__ __forceinline__ float rescaled(Stats p, float m, float c) {
    return p.m == -INFINITY && p.s == 0.0f ? 0.0f : p.s * power(p.m, m, c);
}

// The maximum or sum of a workgroup's floats, to every thread.
template <int B, typename Op>
__device__ __forceinline__ float block_join(float v, Op op) {
    v = lanes_join<64>(v, op);
    if constexpr (B == 64) return v;
    __shared__ float part[B / 64];
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int w = 1; w < B / 64; ++w) s = op(s, part[w]);
    __syncthreads();
    return s;
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

// The position's token, or -1 where it is left out; its weight.
__device__ __forceinline__ int take_token(const PolicyArgs &a, int64_t row, float &weight) {
    weight = a.sums != nullptr ? a.weight[row] : 1.0f;
    return weight == 0.0f ? -1 : a.tokens.get(row, a.vocab);
}

struct Scratch {
    double *terms;   // [3][rows]
    Stats *stats;    // [rows][parts]
    float *at;       // [rows]: the token's logit
};

// N = E::V elements i, i + 1, ... of a row of n; fill past its end.
template <typename E, Use USE>
__device__ __forceinline__ void load_part(Ptr<E> row, int64_t i, int64_t n, float fill,
                                          float (&x)[E::V]) {
    if (i + E::V <= n) {
        E::unpack(load_vec<E, USE>(row + i), x);
        return;
    }
#pragma unroll
    for (int j = 0; j < E::V; ++j) x[j] = i + j < n ? E::get(row[i + j]) : fill;
}

// Maximum and sum of every part of a row, and the token's logit.
template <typename E>
__global__ __launch_bounds__(kBlock) void part_stats_kernel(PolicyArgs a, Scratch w, int64_t parts,
                                                            float c, int64_t first) {
    constexpr int V = E::V, R = kLogitPart / (kBlock * V);
    const int64_t item = first + blockIdx.x;
    const int64_t row = item / parts, at = item % parts * kLogitPart;
    float weight;
    const int token = take_token(a, row, weight);
    if (token < 0) return;
    const Ptr<E> z = (Ptr<E>)a.logits + row * a.ld;
    float x[R][V];
    float m = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; ++r)
        load_part<E, Use::Again>(z, at + (r * kBlock + (int)threadIdx.x) * V, a.vocab, -INFINITY,
                                 x[r]);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) m = fmaxf(m, x[r][j]);
    m = block_join<kBlock>(m, Max());
    // a part of -inf alone: differences from 0, which count nothing
    const float from = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) s += power(x[r][j], from, c);
    s = block_join<kBlock>(s, Sum());
    if (threadIdx.x != 0) return;
    w.stats[item] = {m, s};
    if (token >= at && token < at + kLogitPart) w.at[row] = E::get(z[token]);
}

// A row's statistics from its parts', to every thread of the workgroup.
__device__ __forceinline__ Stats join_parts(const Stats *p, int64_t parts, float c) {
    float m = -INFINITY, s = 0.0f;
    for (int64_t i = threadIdx.x; i < parts; i += kBlock) m = fmaxf(m, p[i].m);
    m = block_join<kBlock>(m, Max());
    for (int64_t i = threadIdx.x; i < parts; i += kBlock) s += rescaled(p[i], m, c);
    return {m, block_join<kBlock>(s, Sum())};
}

// log p of the token from the row's statistics.
__device__ __forceinline__ float log_prob(const PolicyArgs &a, float z, Stats st) {
    return (float)((double)(z - st.m) * a.inv_temperature - (double)logf(st.s));
}

// The gradient of one part of a row; the first part's workgroup writes what
// the row adds to the sums.
template <typename E>
__global__ __launch_bounds__(kBlock) void part_grad_kernel(PolicyArgs a, Scratch w, int64_t parts,
                                                           int64_t grads, float c, int64_t first) {
    constexpr int V = E::V, R = kLogitPart / (kBlock * V);
    const int64_t item = first + blockIdx.x;   // (row, one of the `grads` parts written)
    const int64_t row = item / grads, part = item % grads, at = part * kLogitPart;
    float weight;
    const int token = take_token(a, row, weight);
    const Ptr<E> z = (Ptr<E>)a.logits + row * a.ld;
    const MutPtr<E> out = (MutPtr<E>)a.grad + row * a.ldg;
    Terms t{0.0f, 0.0f, 0.0f, 0.0f};
    Stats st{0.0f, 1.0f};
    float lp = 0.0f, p = 0.0f;
    if (token >= 0) {
        st = join_parts(w.stats + row * parts, parts, c);
        lp = log_prob(a, w.at[row], st);
        p = power(w.at[row], st.m, c) / st.s;
        if (a.sums != nullptr) t = terms_of(a, row, weight, lp);
    }
    if (part == 0 && threadIdx.x == 0) {
        a.logps[row] = lp;
        if (a.sums != nullptr) {
            w.terms[row] = (double)weight * t.loss;
            w.terms[a.rows + row] = (double)weight * t.kl;
            w.terms[2 * a.rows + row] = (double)weight * t.cut;
            if (token < 0)
                for (int k = 0; k < 3; ++k) w.terms[k * a.rows + row] = 0.0;
        }
    }
    if (a.grad == nullptr) return;
    const float by = -t.coef / st.s;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t i = at + (r * kBlock + (int)threadIdx.x) * V;
        if (i >= a.vocab) continue;
        float x[V] = {};
        if (token >= 0) {
            load_part<E, Use::Once>(z, i, a.vocab, 0.0f, x);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[j] = power(x[j], st.m, c) * by;
                if (i + j == token) x[j] = t.coef * (1.0f - p);
            }
        }
        if (i + V <= a.vocab) {
            store_vec<E, Use::Once>(out + i, E::pack(x));
            continue;
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (i + j < a.vocab) out[i + j] = E::put(x[j]);
    }
}

// The loss and the two other sums, in fp64 and a fixed order.
__global__ __launch_bounds__(1024) void sum_terms_kernel(const double *terms, int64_t rows,
                                                         float *sums) {
    for (int k = 0; k < 3; ++k) {
        double s = 0.0;
        for (int64_t i = threadIdx.x; i < rows; i += 1024) s += terms[k * rows + i];
        s = block_sum<1024>(s);
        if (threadIdx.x == 0) sums[k] = (float)s;
    }
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

template <typename E>
hipError_t start_policy(const PolicyArgs &a, hipStream_t s) {
    const PolicyPlan plan = policy_plan(a.rows, a.vocab);
    char *const ws = (char *)a.ws;
    const Scratch w{(double *)(ws + plan.terms), (Stats *)(ws + plan.stats),
                    (float *)(ws + plan.at)};
    const float c = (float)(1.4426950408889634 * a.inv_temperature);
    hipError_t e = over_blocks(a.rows * plan.parts, [&](int64_t first, unsigned n) {
        part_stats_kernel<E><<<n, kBlock, 0, s>>>(a, w, plan.parts, c, first);
    });
    if (e != hipSuccess) return e;
    const int64_t grads = a.grad != nullptr && plan.parts > 0 ? plan.parts : 1;
    e = over_blocks(a.rows * grads, [&](int64_t first, unsigned n) {
        part_grad_kernel<E><<<n, kBlock, 0, s>>>(a, w, plan.parts, grads, c, first);
    });
    if (e != hipSuccess || a.sums == nullptr) return e;
    sum_terms_kernel<<<1, 1024, 0, s>>>(w.terms, a.rows, a.sums);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_policy(const PolicyArgs &a, hipStream_t s) {
    if (a.dtype == ASPIS_F32) return start_policy<F32>(a, s);
    if (a.dtype == ASPIS_BF16) return start_policy<BF16>(a, s);
    return start_policy<F16>(a, s);
}

}  // namespace aspis
