// aspis_tokens.h -- launchers shared by the host entry points of the token
// operators (aspis_tokens.cpp) and their kernels (aspis_tokens.hip,
// aspis_policy.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/aspis.h"

namespace aspis {

// n tokens in memory, int32 or int64.
struct Tokens {
    const void *at;
    int wide;   // int64
#ifdef __HIPCC__
    // Token i, or -1 where it is outside [0, vocab).
    __device__ __forceinline__ int get(int64_t i, int64_t vocab) const {
        const int64_t t = wide ? ((const int64_t *)at)[i] : ((const int32_t *)at)[i];
        return t >= 0 && t < vocab ? (int)t : -1;
    }
#endif
};

constexpr int64_t kMaxVocab = INT32_MAX;          // rows of a table
constexpr int64_t kMaxTokens = int64_t(1) << 30;  // of one embedding gradient, rows of logits

struct EmbedArgs {
    const void *table;
    int64_t vocab, d, ld;
    int dtype;
    Tokens tokens;
    int64_t n;
    float scale;
    void *out;
    int64_t ldo;
    int out_dtype;
};
hipError_t launch_embed(const EmbedArgs &a, hipStream_t s);

// Whether a gradient takes one launch, each workgroup searching all tokens for
// its rows': not where many tokens meet in a row, whose workgroup the others
// would wait for.  In one launch and by sorting, rows of 512, us: 200 tokens
// into 2 rows 14.1 and 14.3, into 16 rows 9.2 and 16.0; 700 into 2 rows 34.1 and
// 14.8, into 64 rows 16.8 and 16.0, into 128 rows 15.4 and 16.6; 1,024 of 2,048
// into 10,000 rows 33.8 and 30.5.
constexpr int kFewTokens = 768;
inline bool embed_few(int64_t n, int64_t vocab) {
    return n <= kFewTokens && (n <= 256 || n <= 8 * vocab);
}
// Otherwise tokens are sorted in runs of kSortRun, kMergeRuns of them merged
// in LDS, longer ones where they are; then the sums of the sorted positions'
// segments, window by window of positions, long ones in pieces of at most a
// block of two windows that are joined afterwards.
constexpr int kSortRun = 1024, kMergeRuns = 32;
// log2 of a window's positions: a function of n alone, since the order of a
// sum follows it.  Small ones give few tokens more waves, large ones cut fewer
// segments.  8 and 32 positions, rows of 2,048 bf16, us: 4,096 tokens 55 and 69,
// 16,384 69 and 77 (into 4 rows 47 and 40), 24,000 82 and 81, 32,768 96 and 88.
inline int embed_shift(int64_t n) { return n <= 16384 ? 3 : 5; }
inline int64_t embed_row(int64_t d) { return (d + 3) / 4 * 4; }   // floats of a partial sum
struct EmbedGradPlan {
    int shift;       // log2 of a window's positions
    int64_t blocks;
    size_t words;    // bytes of an array of n words, and 8 that may be read past them
    size_t bytes;    // four of them (tokens and positions, twice), two partial sums a block
};
inline EmbedGradPlan embed_grad_plan(int64_t n, int64_t d) {
    EmbedGradPlan p;
    p.shift = embed_shift(n);
    p.blocks = (n + (2 << p.shift) - 1) / (2 << p.shift);
    p.words = (size_t)((n + 3) / 4 * 16 + 32);
    p.bytes = 4 * p.words + (size_t)(p.blocks * 2 * embed_row(d)) * sizeof(float);
    return p;
}
struct EmbedGradArgs {
    const void *grad;
    int64_t n, d, ld;
    int dtype;
    Tokens tokens;
    float scale;
    void *out;
    int64_t vocab, ldo;
    int out_dtype;
    bool accumulate;
    void *ws;
};
hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t s);

struct DropoutArgs {
    const void *x;
    int64_t rows, d, ld;
    int dtype;
    uint32_t limit;            // kept: 16 bits >= limit
    float scale;
    uint64_t seed;
    const uint64_t *seed_at;   // or nullptr
    uint64_t offset;
    const void *residual;      // or nullptr
    int64_t ldr;
    void *out;
    int64_t ldo;
};
hipError_t launch_dropout(const DropoutArgs &a, hipStream_t s);

constexpr int64_t kMaxLogits = int64_t(1) << 24;
// How a row of so many 16-byte vectors is held by `lanes` lanes of `vecs` each,
// and into how many units that cuts it: by its length alone.
constexpr int kBlockVecs = 1024 * 16;
struct PolicyCut {
    int lanes, vecs, units;
};
inline PolicyCut policy_cut(int64_t nv) {
    const int cuts[][2] = {{64, 1},  {64, 2},   {64, 4},   {64, 8},   {256, 4},   {256, 6},   {256, 8},
                           {256, 10}, {256, 16}, {512, 10}, {512, 16}, {1024, 10}, {1024, 12}};
    for (const auto &c : cuts)
        if (nv <= c[0] * c[1]) return {c[0], c[1], c[0] / 64 * (c[1] > 8 ? 2 : 1)};
    return {1024, 16, (int)((nv + kBlockVecs - 1) / kBlockVecs) * 32};
}
// Workgroups that add up the rows' terms, before one joins theirs.
inline int sum_groups(int64_t rows) {
    return rows <= 8192 ? 1 : rows >= 64 * 4096 ? 64 : (int)((rows + 4095) / 4096);
}
struct PolicyPlan {
    int units;                          // of a row
    size_t terms, partial, stats, at;   // offsets of the workspace's arrays
    size_t bytes;
};
inline PolicyPlan policy_plan(int64_t rows, int64_t vocab, int elem_bytes) {
    PolicyPlan p;
    p.units = policy_cut((vocab * elem_bytes + 15) / 16).units;
    p.terms = 0;                                   // double [3][rows], then [3][sum_groups]
    p.partial = p.terms + (size_t)rows * 3 * sizeof(double);
    p.stats = p.partial + (size_t)sum_groups(rows) * 3 * sizeof(double);   // float2 [rows][units]
    p.at = p.stats + (size_t)(rows * p.units) * 8;          // float [rows]
    p.bytes = (p.at + (size_t)rows * 4 + 15) / 16 * 16;
    return p;
}
struct PolicyArgs {
    const void *logits;
    int64_t rows, vocab, ld;
    int dtype;
    Tokens tokens;
    double inv_temperature;
    // the loss; sums == nullptr: log-probabilities alone
    const float *old, *advantage, *weight, *ref;
    float clip_low, clip_high, kl;   // the borders 1 - low and 1 + high
    float grad_scale;                // over the temperature
    float *sums, *logps;
    void *grad;                      // or nullptr
    int64_t ldg;
    void *ws;
};
hipError_t launch_policy(const PolicyArgs &a, hipStream_t s);

}  // namespace aspis
