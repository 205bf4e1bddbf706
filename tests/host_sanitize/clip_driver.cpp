// The host side of the norm, clipping and update operators under the
// sanitizers: tables, row plans and the entry points' checks, with launchers
// that fail.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2108_02416_amd/csrc/aspis_clip.h"

namespace aspis {
hipError_t launch_norm(const aspis_chunk *, int64_t, int32_t, double *, NormIn, float *,
                       hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_clip(const aspis_chunk *, const aspis_chunk *, int64_t, bool, double *, NormIn,
                       hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_sgd(const aspis_chunk *, const aspis_chunk *, const aspis_chunk *,
                      const aspis_chunk *, int64_t, bool, double *, const NormIn &, const SgdArgs &,
                      bool, hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_adamw(const aspis_chunk *, const aspis_chunk *, const aspis_chunk *,
                        const aspis_chunk *, const aspis_chunk *, int64_t, bool, double *,
                        const NormIn &, const AdamArgs &, bool, hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_rows(const RowArgs &, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace aspis

#define CHECK(x)                                                          \
    do {                                                                  \
        if (!(x)) {                                                       \
            std::printf("failed: %s (line %d)\n", #x, __LINE__);          \
            std::exit(1);                                                 \
        }                                                                 \
    } while (0)

static void check_plan(int64_t rows, int64_t d, int elem) {
    const aspis::RowPlan p = aspis::row_plan(rows, d, elem);
    const int64_t v = 16 / elem, nv = (d + v - 1) / v;
    if (p.kind == aspis::RowKind::Registers) {
        CHECK(nv <= aspis::kRowVecs && p.scratch == 0);
        return;
    }
    CHECK(nv > aspis::kRowVecs);
    CHECK(p.parts >= 1 && p.parts <= 1024 && p.length >= 1);
    // every element is in one part, and no part is empty
    CHECK((int64_t)p.parts * p.length >= d && (int64_t)(p.parts - 1) * p.length < d);
    // the order of the sum depends on the length of a row alone
    const aspis::RowPlan one = aspis::row_plan(1, d, elem), many = aspis::row_plan(100000, d, elem);
    CHECK(one.parts == p.parts && one.length == p.length);
    CHECK(many.parts == p.parts && many.length == p.length);
    if (p.kind == aspis::RowKind::Parts) {
        CHECK((p.vecs == 8 || p.vecs == 24) && p.length <= 256 * p.vecs * v);
        CHECK(p.length % (256 * v) == 0);
        // sums, a line each for totals and arrivals, the list of parts
        CHECK(p.scratch * 8 >= rows * (p.parts * 8 + 256) + (rows * p.parts + 1) * 4);
    } else {
        CHECK(p.scratch >= rows * p.parts);
    }
}

int main() {
    for (int elem : {2, 4})
        for (int64_t rows : {int64_t(1), int64_t(3), int64_t(100), int64_t(6900)})
            for (int64_t d = 1; d < aspis::kMaxRow; d += 1 + d / 7)
                for (int64_t off : {-1, 0, 1})
                    if (d + off >= 1) check_plan(rows, d + off, elem);

    std::vector<int64_t> numel = {0, 1, 4095, 4096, 4097, 0, 1000000};
    std::vector<int32_t> type = {0, 1, 2, 0, 1, 2, 0};
    std::vector<const void *> ptr(numel.size());
    for (size_t i = 0; i < ptr.size(); ++i)
        ptr[i] = numel[i] ? reinterpret_cast<const void *>((uintptr_t)(i + 1) << 32) : nullptr;
    const int n = (int)numel.size();
    const int64_t entries = aspis_tensor_entries(numel.data(), n);
    CHECK(entries == aspis_tensor_chunks(numel.data(), n) + n);
    std::vector<aspis_chunk> table((size_t)entries);   // exactly as many as the table needs
    CHECK(aspis_tensor_table(ptr.data(), numel.data(), type.data(), n, table.data(), entries) ==
          ASPIS_OK);
    CHECK(aspis_tensor_table(ptr.data(), numel.data(), type.data(), n, table.data(), entries - 1) ==
          ASPIS_ERR_BUFFER_SMALL);

    alignas(16) static char ws[1 << 16];
    alignas(16) static aspis_chunk dummy[4];
    double sumsq = 0;
    float norm = 0;
    CHECK(aspis_grad_norm(dummy, 2, 1, &sumsq, &norm, nullptr, ws, sizeof ws, nullptr) ==
          ASPIS_ERR_DEVICE);
    CHECK(aspis_clip_grads(dummy, nullptr, 2, 1.0, &sumsq, &norm, 0, ws, sizeof ws, nullptr) ==
          ASPIS_ERR_DEVICE);
    aspis_sgd sgd = {0.1, 0.9, 0.0, 1.0, 1, 0};
    CHECK(aspis_clipped_sgd(dummy, dummy, dummy, nullptr, 2, &sgd, &sumsq, &norm, ws, sizeof ws,
                            nullptr) == ASPIS_ERR_DEVICE);
    CHECK(aspis_clipped_sgd(dummy, dummy, dummy, nullptr, 2, nullptr, &sumsq, &norm, ws, sizeof ws,
                            nullptr) == ASPIS_ERR_INVALID_ARG);
    aspis_adamw adam = {0.1, 0.9, 0.99, 1e-8, 0.0, 1.0, 1, 0, 0};
    CHECK(aspis_clipped_adamw(dummy, dummy, dummy, dummy, nullptr, 2, &adam, &sumsq, &norm, ws,
                              sizeof ws, nullptr) == ASPIS_ERR_DEVICE);
    CHECK(aspis_clipped_adamw(dummy, dummy, dummy, dummy, nullptr, 2, nullptr, &sumsq, &norm, ws,
                              sizeof ws, nullptr) == ASPIS_ERR_INVALID_ARG);
    float rows[64];
    CHECK(aspis_row_norms(rows, 4, 8, 8, ASPIS_F32, &norm, nullptr, 0, nullptr) == ASPIS_ERR_DEVICE);
    CHECK(aspis_clip_rows(rows, 4, 8, 8, ASPIS_F32, 1.0, rows, 8, nullptr, 0, nullptr, 0, nullptr) ==
          ASPIS_ERR_DEVICE);
    CHECK(aspis_last_error()[0] != 0);
    std::printf("ok\n");
    return 0;
}
