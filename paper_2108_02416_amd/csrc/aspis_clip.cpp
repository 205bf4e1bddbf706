// aspis_clip.cpp -- C ABI of the norm, clipping and update operators:
// argument checking, tensor tables, workspaces and launches (the kernels are
// in aspis_clip.hip).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/aspis.h"
#include "aspis_clip.h"

namespace aspis {
aspis_status host_fail(aspis_status st, const char *msg);   // aspis_host.cpp
void host_clear_error();

RowPlan row_plan(int64_t rows, int64_t d, int elem_bytes) {
    const int64_t per_vec = 16 / elem_bytes, nv = (d + per_vec - 1) / per_vec;
    if (nv <= kRowVecs) return {RowKind::Registers, 0, 1, 0, 0};
    RowPlan p{RowKind::Parts, 8, 0, 0, 0};
    auto parts = [&](int64_t vecs) { return (nv + 256 * vecs - 1) / (256 * vecs); };
    // Registers hold 64 MB of parts of 8 vectors a thread at once, 96 MB of 24.
    // Rows of 300,000 f32: 45.6 us of 100 with 8, 50.5 with 24; rows of
    // 5 million: 306 us of 40 with 8, 272 with 24.
    if (parts(8) > 128) p.vecs = 24;
    int64_t step = 256 * per_vec, n = parts(p.vecs);
    if (n > 768) {
        // More than three quarters of the 1,024 workgroups that run at once:
        // the row goes by segment_kernel, in at most 1,024 parts of whole
        // chunks, since all its sums are read by all that scale it.
        p.kind = RowKind::Segments;
        step = kChunk;
        n = 1024;
    }
    // Up to 16 MB two launches over the cache take less than three: 40 rows of
    // 100,000 f32 14.5 against 17.8 us, 20 of 400,000 20.0 against 18.3.
    if (rows * d * elem_bytes < (int64_t)16 << 20) p.kind = RowKind::Segments;
    // parts of about the same length, in whole vectors of all 256 threads
    const int64_t length = (d + n * step - 1) / (n * step) * step;
    p.length = (int32_t)length;
    p.parts = (int32_t)((d + length - 1) / length);
    // a row's sums; for parts that wait for one another also a line each for
    // its total and its arrivals, and a list of parts in 32-bit words
    p.scratch = rows * p.parts;
    if (p.kind == RowKind::Parts) p.scratch += rows * 32 + (rows * p.parts + 2) / 2;
    return p;
}
}  // namespace aspis

namespace {

using aspis::host_fail;

constexpr int64_t kMaxElements = int64_t(1) << 60;

aspis_status fail(aspis_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
aspis_status fail(aspis_status st, const char *fmt, ...) {
    char msg[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return host_fail(st, msg);
}

aspis_status launched(hipError_t e, const char *what) {
    if (e != hipSuccess)
        return fail(ASPIS_ERR_DEVICE, "%s failed: %s", what, hipGetErrorString(e));
    aspis::host_clear_error();
    return ASPIS_OK;
}

int elem_bytes(int dtype) {
    return dtype == ASPIS_F32 ? 4 : dtype == ASPIS_BF16 || dtype == ASPIS_F16 ? 2 : 0;
}

// Chunks of a list: -1 on invalid sizes, -2 past the limits.
int64_t count_chunks(const int64_t *numel, int32_t count) {
    if (count < 0 || (count > 0 && numel == nullptr)) return -1;
    if (count > aspis::kMaxTensors) return -2;
    int64_t n = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (numel[i] < 0) return -1;
        if (numel[i] > kMaxElements) return -2;
        n += aspis::chunks_of(numel[i]);
        if (n > aspis::kMaxChunks) return -2;
    }
    return n;
}

size_t list_workspace(int64_t n_chunks) {
    return (size_t)aspis::norm_doubles(n_chunks) * sizeof(double);
}

aspis_status check_list(const char *who, const void *table, int64_t n_chunks, double max_norm,
                        const double *sumsq, const float *norm, const void *ws, size_t ws_bytes) {
    if (n_chunks < 0 || n_chunks > aspis::kMaxChunks)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: n_chunks=%lld", who, (long long)n_chunks);
    if (n_chunks > 0 && table == nullptr)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL table", who);
    if (sumsq == nullptr || norm == nullptr)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: sumsq and norm must be non-NULL", who);
    if (!(max_norm >= 0.0))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: max_norm=%g must be >= 0", who, max_norm);
    if (((uintptr_t)table | (uintptr_t)ws) % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: tables and workspace must be 16-byte aligned", who);
    if (n_chunks > 0 && (ws == nullptr || ws_bytes < list_workspace(n_chunks)))
        return fail(ASPIS_ERR_BUFFER_SMALL, "%s: workspace of %zu bytes, %zu needed", who,
                    ws == nullptr ? (size_t)0 : ws_bytes, list_workspace(n_chunks));
    return ASPIS_OK;
}

aspis_status check_rows(const char *who, const void *x, int64_t rows, int64_t d, int64_t ld,
                        int dtype, const void *ws, size_t ws_bytes) {
    const int size = elem_bytes(dtype);
    if (size == 0) return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown type %d", who, dtype);
    if (rows < 0 || d < 0 || ld < d)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: rows=%lld d=%lld ld=%lld", who, (long long)rows,
                    (long long)d, (long long)ld);
    if (d > aspis::kMaxRow || (rows > 0 && ld > kMaxElements / rows))
        return fail(ASPIS_ERR_OVERFLOW, "%s: d=%lld or rows * ld is too large", who, (long long)d);
    if (rows > 0 && d > 0 && (x == nullptr || (uintptr_t)x % size != 0))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL or misaligned rows", who);
    const size_t need = aspis_row_workspace(rows, d, (aspis_dtype)dtype);
    if (need > 0 && (ws == nullptr || ws_bytes < need))
        return fail(ASPIS_ERR_BUFFER_SMALL, "%s: workspace of %zu bytes, %zu needed", who,
                    ws == nullptr ? (size_t)0 : ws_bytes, need);
    if ((uintptr_t)ws % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
    return ASPIS_OK;
}

aspis_status check_update(const char *who, const void *const *tables, int n_tables,
                          int64_t n_chunks, uint32_t flags) {
    for (int i = 0; i < n_tables; ++i)
        if (n_chunks > 0 && tables[i] == nullptr)
            return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL table", who);
    for (int i = 0; i < n_tables; ++i)
        if ((uintptr_t)tables[i] % 16 != 0)
            return fail(ASPIS_ERR_INVALID_ARG, "%s: tables must be 16-byte aligned", who);
    if (flags & ~(ASPIS_CLIP_HAVE_SUMSQ | ASPIS_CLIP_SKIP_NONFINITE))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", who, flags);
    return ASPIS_OK;
}

}  // namespace

extern "C" {

int64_t aspis_tensor_chunks(const int64_t *numel, int32_t count) {
    const int64_t n = count_chunks(numel, count);
    return n < 0 ? -1 : n;
}

int64_t aspis_tensor_entries(const int64_t *numel, int32_t count) {
    const int64_t n = count_chunks(numel, count);
    return n < 0 ? -1 : n + count;
}

aspis_status aspis_tensor_table(const void *const *ptr, const int64_t *numel,
                                const int32_t *dtype, int32_t count, aspis_chunk *table,
                                int64_t cap) {
    const int64_t chunks = count_chunks(numel, count);
    if (chunks == -2) return fail(ASPIS_ERR_OVERFLOW, "aspis_tensor_table: too many elements");
    if (chunks < 0) return fail(ASPIS_ERR_INVALID_ARG, "aspis_tensor_table: negative size or NULL");
    if (count > 0 && (ptr == nullptr || dtype == nullptr || table == nullptr))
        return fail(ASPIS_ERR_INVALID_ARG, "aspis_tensor_table: NULL argument");
    for (int32_t i = 0; i < count; ++i) {
        const int size = elem_bytes(dtype[i]);
        if (size == 0)
            return fail(ASPIS_ERR_INVALID_ARG, "aspis_tensor_table: tensor %d has unknown type %d",
                        i, dtype[i]);
        if (numel[i] > 0 && (ptr[i] == nullptr || (uintptr_t)ptr[i] % size != 0))
            return fail(ASPIS_ERR_INVALID_ARG, "aspis_tensor_table: tensor %d is NULL or misaligned",
                        i);
    }
    if (cap < chunks + count)
        return fail(ASPIS_ERR_BUFFER_SMALL, "need %lld entries, buffer holds %lld",
                    (long long)(chunks + count), (long long)cap);
    int64_t k = 0;
    int32_t filled = 0;   // tensors before this one that are not empty
    for (int32_t i = 0; i < count; ++i) {
        const int size = elem_bytes(dtype[i]);
        table[chunks + i] = {(uint64_t)k, (int32_t)aspis::chunks_of(numel[i]), filled};
        for (int64_t at = 0; at < numel[i]; at += aspis::kChunk) {
            const int64_t left = numel[i] - at;
            table[k++] = {(uint64_t)(uintptr_t)ptr[i] + (uint64_t)(at * size),
                          (int32_t)(left < aspis::kChunk ? left : aspis::kChunk),
                          filled * 4 + dtype[i]};
        }
        filled += numel[i] > 0;
    }
    aspis::host_clear_error();
    return ASPIS_OK;
}

size_t aspis_norm_workspace(int64_t n_chunks) {
    if (n_chunks < 0 || n_chunks > aspis::kMaxChunks) return 0;
    return list_workspace(n_chunks);
}

aspis_status aspis_grad_norm(const aspis_chunk *table, int64_t n_chunks, int32_t n_tensors,
                             double *sumsq, float *norm, float *each, void *workspace,
                             size_t ws_bytes, void *stream) {
    const char *who = "aspis_grad_norm";
    aspis_status st = check_list(who, table, n_chunks, 0.0, sumsq, norm, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    if (n_tensors < 0 || n_tensors > aspis::kMaxTensors || (each != nullptr && n_tensors > 0 && table == nullptr))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: n_tensors=%d or NULL table", who, n_tensors);
    const aspis::NormIn in{nullptr, 0, sumsq, norm, 0.0};
    return launched(aspis::launch_norm(table, n_chunks, n_tensors, static_cast<double *>(workspace),
                                       in, each, static_cast<hipStream_t>(stream)),
                    who);
}

aspis_status aspis_clip_grads(const aspis_chunk *table, const aspis_chunk *out_table,
                              int64_t n_chunks, double max_norm, double *sumsq, float *norm,
                              uint32_t flags, void *workspace, size_t ws_bytes, void *stream) {
    const char *who = "aspis_clip_grads";
    aspis_status st = check_list(who, table, n_chunks, max_norm, sumsq, norm, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    if (flags & ~ASPIS_CLIP_HAVE_SUMSQ)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", who, flags);
    if ((uintptr_t)out_table % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: tables must be 16-byte aligned", who);
    const aspis::NormIn in{nullptr, 0, sumsq, norm, max_norm};
    return launched(aspis::launch_clip(table, out_table == table ? nullptr : out_table, n_chunks,
                                       (flags & ASPIS_CLIP_HAVE_SUMSQ) != 0,
                                       static_cast<double *>(workspace), in,
                                       static_cast<hipStream_t>(stream)),
                    who);
}

size_t aspis_row_workspace(int64_t rows, int64_t d, aspis_dtype dtype) {
    const int size = elem_bytes(dtype);
    if (size == 0 || rows < 0 || d < 0 || d > aspis::kMaxRow ||
        (rows > 0 && d > kMaxElements / rows))
        return SIZE_MAX;
    return (size_t)aspis::row_plan(rows, d, size).scratch * sizeof(double);
}

aspis_status aspis_row_norms(const void *x, int64_t rows, int64_t d, int64_t ld,
                             aspis_dtype dtype, float *norms, void *workspace, size_t ws_bytes,
                             void *stream) {
    const char *who = "aspis_row_norms";
    const aspis_status st = check_rows(who, x, rows, d, ld, dtype, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    if (rows > 0 && norms == nullptr) return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL norms", who);
    const aspis::RowArgs a{x, nullptr, norms, rows, d, ld, ld, dtype, 0.0,
                           static_cast<double *>(workspace), false};
    return launched(aspis::launch_rows(a, static_cast<hipStream_t>(stream)), who);
}

aspis_status aspis_clip_rows(const void *x, int64_t rows, int64_t d, int64_t ld,
                             aspis_dtype dtype, double max_norm, void *out, int64_t ldo,
                             float *norms, uint32_t flags, void *workspace, size_t ws_bytes,
                             void *stream) {
    const char *who = "aspis_clip_rows";
    const aspis_status st = check_rows(who, x, rows, d, ld, dtype, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    if (!(max_norm >= 0.0))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: max_norm=%g must be >= 0", who, max_norm);
    if (flags & ~ASPIS_CLIP_NO_WAIT)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", who, flags);
    const int size = elem_bytes(dtype);
    if (ldo < d || (rows > 0 && ldo > kMaxElements / rows))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: ldo=%lld", who, (long long)ldo);
    if (rows > 0 && d > 0) {
        if (out == nullptr || (uintptr_t)out % size != 0)
            return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL or misaligned out", who);
        const uintptr_t x0 = (uintptr_t)x, o0 = (uintptr_t)out;
        const uintptr_t x1 = x0 + (uintptr_t)(((rows - 1) * ld + d) * size);
        const uintptr_t o1 = o0 + (uintptr_t)(((rows - 1) * ldo + d) * size);
        const bool same = x0 == o0 && (ld == ldo || rows == 1);
        if (!same && x0 < o1 && o0 < x1)
            return fail(ASPIS_ERR_INVALID_ARG, "%s: out overlaps x without being x", who);
    }
    const aspis::RowArgs a{x, out, norms, rows, d, ld, ldo, dtype, max_norm,
                           static_cast<double *>(workspace), (flags & ASPIS_CLIP_NO_WAIT) == 0};
    return launched(aspis::launch_rows(a, static_cast<hipStream_t>(stream)), who);
}

aspis_status aspis_clipped_sgd(const aspis_chunk *params, const aspis_chunk *grads,
                               const aspis_chunk *mean, const aspis_chunk *copies,
                               int64_t n_chunks, const aspis_sgd *opt, double *sumsq, float *norm,
                               void *workspace, size_t ws_bytes, void *stream) {
    const char *who = "aspis_clipped_sgd";
    if (opt == nullptr) return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL options", who);
    aspis_status st =
        check_list(who, grads, n_chunks, opt->max_norm, sumsq, norm, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    const void *needed[] = {params, opt->momentum != 0.0 ? mean : params};
    st = check_update(who, needed, 2, n_chunks, opt->flags);
    if (st != ASPIS_OK) return st;
    if (((uintptr_t)mean | (uintptr_t)copies) % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: tables must be 16-byte aligned", who);
    if (!std::isfinite(opt->lr) || !(opt->momentum >= 0.0 && opt->momentum < 1.0) ||
        !(opt->weight_decay >= 0.0 && std::isfinite(opt->weight_decay)))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: lr=%g momentum=%g weight_decay=%g", who, opt->lr,
                    opt->momentum, opt->weight_decay);
    const aspis::NormIn in{nullptr, 0, sumsq, norm, opt->max_norm};
    const aspis::SgdArgs a{(float)opt->lr, (float)opt->momentum, (float)opt->weight_decay,
                           opt->nesterov != 0};
    return launched(aspis::launch_sgd(params, grads, mean, copies, n_chunks,
                                      (opt->flags & ASPIS_CLIP_HAVE_SUMSQ) != 0,
                                      static_cast<double *>(workspace), in, a,
                                      (opt->flags & ASPIS_CLIP_SKIP_NONFINITE) != 0,
                                      static_cast<hipStream_t>(stream)),
                    who);
}

aspis_status aspis_clipped_adamw(const aspis_chunk *params, const aspis_chunk *grads,
                                 const aspis_chunk *mean, const aspis_chunk *square,
                                 const aspis_chunk *copies, int64_t n_chunks,
                                 const aspis_adamw *opt, double *sumsq, float *norm,
                                 void *workspace, size_t ws_bytes, void *stream) {
    const char *who = "aspis_clipped_adamw";
    if (opt == nullptr) return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL options", who);
    aspis_status st =
        check_list(who, grads, n_chunks, opt->max_norm, sumsq, norm, workspace, ws_bytes);
    if (st != ASPIS_OK) return st;
    const void *needed[] = {params, mean, square};
    st = check_update(who, needed, 3, n_chunks, opt->flags);
    if (st != ASPIS_OK) return st;
    if ((uintptr_t)copies % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: tables must be 16-byte aligned", who);
    if (!std::isfinite(opt->lr) || !(opt->beta_one >= 0.0 && opt->beta_one < 1.0) ||
        !(opt->beta_two >= 0.0 && opt->beta_two < 1.0) ||
        !(opt->eps >= 0.0 && std::isfinite(opt->eps)) ||
        !(opt->weight_decay >= 0.0 && std::isfinite(opt->weight_decay)) || opt->step < 1)
        return fail(ASPIS_ERR_INVALID_ARG,
                    "%s: lr=%g beta_one=%g beta_two=%g eps=%g weight_decay=%g step=%lld", who,
                    opt->lr, opt->beta_one, opt->beta_two, opt->eps, opt->weight_decay,
                    (long long)opt->step);
    const aspis::NormIn in{nullptr, 0, sumsq, norm, opt->max_norm};
    // the constants of a step, each rounded to f32 once
    const double t = (double)opt->step;
    const aspis::AdamArgs a{(float)(1.0 - opt->lr * opt->weight_decay),
                            (float)opt->beta_one,
                            (float)(1.0 - opt->beta_one),
                            (float)opt->beta_two,
                            (float)(1.0 - opt->beta_two),
                            (float)(opt->lr / (1.0 - std::pow(opt->beta_one, t))),
                            (float)(1.0 / std::sqrt(1.0 - std::pow(opt->beta_two, t))),
                            (float)opt->eps};
    return launched(aspis::launch_adamw(params, grads, mean, square, copies, n_chunks,
                                        (opt->flags & ASPIS_CLIP_HAVE_SUMSQ) != 0,
                                        static_cast<double *>(workspace), in, a,
                                        (opt->flags & ASPIS_CLIP_SKIP_NONFINITE) != 0,
                                        static_cast<hipStream_t>(stream)),
                    who);
}

}  // extern "C"
