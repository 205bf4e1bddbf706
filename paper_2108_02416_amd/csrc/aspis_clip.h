// aspis_clip.h -- launchers shared by the host entry points of the norm,
// clipping and update operators (aspis_clip.cpp) and their kernels
// (aspis_clip.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/aspis.h"

namespace aspis {

// Elements per chunk of a tensor list: a workgroup's unit of work.
constexpr int kChunk = 16384;
// aspis_chunk.info of a chunk: the tensor's aspis_dtype.  The table's
// n_tensors further entries give tensor t's chunks: addr = the first one's
// index, n = their number.
inline int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }

// Workgroups of the norm pass over a list, and so its partial sums: a
// function of the list alone, since the order of the sum follows it.
constexpr int kNormGroups = 2048;
inline int norm_groups(int64_t n_chunks) {
    return (int)(n_chunks < kNormGroups ? n_chunks : kNormGroups);
}

// The global norm's inputs to a kernel that applies it: n_partial sums of
// squares (0: the sum is in *sumsq already), and where the results go.
struct NormIn {
    const double *partial;
    int n_partial;
    double *sumsq;
    float *norm;
    double max_norm;
};

hipError_t launch_list_sumsq(const aspis_chunk *table, int64_t n_chunks, double *partial,
                             double *chunk_sums, hipStream_t s);
hipError_t launch_list_norm(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors,
                            const NormIn &in, const double *chunk_sums, float *each,
                            hipStream_t s);
hipError_t launch_list_scale(const aspis_chunk *table, const aspis_chunk *out, int64_t n_chunks,
                             const NormIn &in, hipStream_t s);

struct SgdArgs {
    float lr, momentum, decay;
    int nesterov;
};
struct AdamArgs {
    float shrink, beta1, rest1, beta2, rest2, step_size, root2, eps;
};
hipError_t launch_sgd(const aspis_chunk *params, const aspis_chunk *grads,
                      const aspis_chunk *mean, const aspis_chunk *copies, int64_t n_chunks,
                      const NormIn &in, const SgdArgs &a, bool skip, hipStream_t s);
hipError_t launch_adamw(const aspis_chunk *params, const aspis_chunk *grads,
                        const aspis_chunk *mean, const aspis_chunk *square,
                        const aspis_chunk *copies, int64_t n_chunks, const NormIn &in,
                        const AdamArgs &a, bool skip, hipStream_t s);

// Rows.  A row of up to kRowVecs 16-byte vectors is held in one workgroup's
// registers; a longer one is cut into segments.
constexpr int kRowVecs = 8192;
struct RowSplit {
    int64_t seg;     // elements per segment (0: the row is not cut)
    int32_t parts;   // segments per row
};
RowSplit row_split(int64_t d, int elem_bytes);
struct RowArgs {
    const void *x;
    void *out;       // nullptr: norms only
    float *norms;    // or nullptr
    int64_t rows, d, ld, ldo;
    int dtype;
    double max_norm;
    double *partial; // [rows][parts], long rows only
};
hipError_t launch_rows(const RowArgs &a, hipStream_t s);

}  // namespace aspis
