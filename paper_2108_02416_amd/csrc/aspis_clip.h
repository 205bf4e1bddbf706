// aspis_clip.h -- launchers shared by the host entry points of the norm,
// clipping and update operators (aspis_clip.cpp) and their kernels
// (aspis_clip.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/aspis.h"

namespace aspis {

// Elements per chunk of a tensor list: a workgroup's unit of work.
constexpr int kChunk = 4096;
// A table holds n_chunks chunks (info: the type, plus 4 times the tensor's
// index among those that are not empty), then an entry per tensor: addr its
// first chunk's index, n its number of chunks, info its index among those
// that are not empty.
inline int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }
constexpr int64_t kMaxChunks = int64_t(1) << 26;    // of a list: 2^38 elements
constexpr int32_t kMaxTensors = 1 << 23;            // a workgroup each (their own norms)
constexpr int64_t kMaxRow = int64_t(1) << 34;       // elements of a row: one launch

// Workgroups of the norm pass over a list, at most, and so its partial sums:
// a function of the list alone, since the order of the sum follows it.
constexpr int kNormGroups = 1024;
// Lists of up to so many chunks are one workgroup's work, longer ones several
// workgroups' in two launches.  Both ways in us, the call included: a norm of
// 16 chunks 5.4 and 7.9; a clip of 8 7.3 and 8.7, of 12 9.6 and 8.7; an AdamW
// update of 4 9.4 and 10.8, of 5 11.2 and 10.8 (SGD: of 4 7.4 and 10.2, of 6
// 9.0 and 10.3, of 8 10.5 and 10.3).
constexpr int kSoloChunks = 16, kSoloClip = 8, kSoloUpdate = 4;
// The workspace of a list, in doubles: the partial sums, then the sums of
// runs of chunks for the tensors' own norms.
inline int64_t norm_doubles(int64_t n_chunks) { return kNormGroups + 2 * n_chunks; }

// The global norm's inputs to a kernel that applies it: n_partial sums of
// squares (0: the sum is in *sumsq already), and where the results go.
struct NormIn {
    const double *partial;
    int n_partial;
    double *sumsq;
    float *norm;
    double max_norm;
};

// ws: norm_doubles(n_chunks) doubles.  have_sumsq: *in.sumsq is given.
hipError_t launch_norm(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors, double *ws,
                       NormIn in, float *each, hipStream_t s);
hipError_t launch_clip(const aspis_chunk *table, const aspis_chunk *out, int64_t n_chunks,
                       bool have_sumsq, double *ws, NormIn in, hipStream_t s);

struct SgdArgs {
    float lr, momentum, decay;
    int nesterov;
};
struct AdamArgs {
    float shrink, beta1, rest1, beta2, rest2, step_size, root2, eps;
};
hipError_t launch_sgd(const aspis_chunk *params, const aspis_chunk *grads,
                      const aspis_chunk *mean, const aspis_chunk *copies, int64_t n_chunks,
                      bool have_sumsq, double *ws, const NormIn &in, const SgdArgs &a, bool skip,
                      hipStream_t s);
hipError_t launch_adamw(const aspis_chunk *params, const aspis_chunk *grads,
                        const aspis_chunk *mean, const aspis_chunk *square,
                        const aspis_chunk *copies, int64_t n_chunks, bool have_sumsq, double *ws,
                        const NormIn &in, const AdamArgs &a, bool skip, hipStream_t s);

// Rows.  How a row is summed depends on its length alone (parts of `length`
// elements), so that its norm does; which kernel clips it also on how many
// there are.
constexpr int kRowVecs = 8192;   // 16-byte vectors of a row that one workgroup holds
enum class RowKind {
    Registers,   // in one workgroup's registers
    Parts,       // in several workgroups' (vecs vectors a thread)
    Segments     // read twice, the second time from the last-level cache
};
struct RowPlan {
    RowKind kind;
    int32_t vecs;            // vectors of a part per thread
    int32_t parts, length;   // of a row; elements of a part
    int64_t scratch;         // doubles of workspace
};
RowPlan row_plan(int64_t rows, int64_t d, int elem_bytes);
struct RowArgs {
    const void *x;
    void *out;       // nullptr: norms only
    float *norms;    // or nullptr
    int64_t rows, d, ld, ldo;
    int dtype;
    double max_norm;
    double *scratch; // row_plan's, 16-byte aligned
    bool wait;       // workgroups may wait for one another
};
hipError_t launch_rows(const RowArgs &a, hipStream_t s);

}  // namespace aspis
