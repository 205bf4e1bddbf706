// aspis_tokens.cpp -- C ABI of the token operators: argument checking,
// workspaces and launches (the kernels are in aspis_tokens.hip and
// aspis_policy.hip).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "../../include/aspis.h"
#include "aspis_errors.h"
#include "aspis_tokens.h"

namespace {

using aspis::elem_bytes;
using aspis::fail;
using aspis::kMaxElements;
using aspis::launched;

// Rows of d elements, ld from one's start to the next's.
struct Rows {
    const char *name;
    const void *at;
    int64_t rows, d, ld;
    int dtype;
    bool empty() const { return rows == 0 || d == 0; }
    uintptr_t begin() const { return (uintptr_t)at; }
    uintptr_t end() const {
        return begin() + (uintptr_t)(((rows - 1) * ld + d) * elem_bytes(dtype));
    }
};

aspis_status check_rows(const char *who, const Rows &x) {
    const int size = elem_bytes(x.dtype);
    if (size == 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: %s: unknown type %d", who, x.name, x.dtype);
    if (x.rows < 0 || x.d < 0 || x.ld < x.d)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: %s: rows=%lld d=%lld ld=%lld", who, x.name,
                    (long long)x.rows, (long long)x.d, (long long)x.ld);
    if (x.rows > 0 && x.ld > kMaxElements / x.rows)
        return fail(ASPIS_ERR_OVERFLOW, "%s: %s: rows * ld is too large", who, x.name);
    if (!x.empty() && (x.at == nullptr || (uintptr_t)x.at % size != 0))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: %s is NULL or misaligned", who, x.name);
    return ASPIS_OK;
}

// n values of `size` bytes, as a row.  (More than memory holds: of no rows, so
// that nothing is written.)
Rows array(const char *name, const void *at, int64_t n, int64_t size) {
    const int64_t d = at != nullptr && n <= kMaxElements / 8 ? (n * size + 3) / 4 : 0;
    return {name, at, 1, d, d, ASPIS_F32};
}

// Whether two sets of rows share memory.  Columns of the same rows do not.
bool overlap(const Rows &a, const Rows &b) {
    if (a.empty() || b.empty() || a.begin() >= b.end() || b.begin() >= a.end()) return false;
    const uintptr_t size_a = elem_bytes(a.dtype), size_b = elem_bytes(b.dtype);
    const uintptr_t pitch = a.ld * size_a;
    if (pitch != b.ld * size_b) return true;
    const bool swap = b.begin() < a.begin();
    const uintptr_t apart = (swap ? a.begin() - b.begin() : b.begin() - a.begin()) % pitch;
    return apart < (swap ? b.d * size_b : a.d * size_a) ||
           apart + (swap ? a.d * size_a : b.d * size_b) > pitch;
}

// Whether they are the same rows.
bool same(const Rows &a, const Rows &b) {
    return a.at == b.at && a.dtype == b.dtype && (a.ld == b.ld || a.rows == 1);
}

// What a call writes shares no memory, nor any with what it reads.
aspis_status check_apart(const char *who, std::initializer_list<Rows> written,
                         std::initializer_list<Rows> read) {
    for (const Rows *w = written.begin(); w != written.end(); ++w) {
        for (const Rows *v = w + 1; v != written.end(); ++v)
            if (overlap(*w, *v))
                return fail(ASPIS_ERR_INVALID_ARG, "%s: %s and %s overlap", who, w->name, v->name);
        for (const Rows &r : read)
            if (overlap(*w, r))
                return fail(ASPIS_ERR_INVALID_ARG, "%s: %s overlaps %s", who, w->name, r.name);
    }
    return ASPIS_OK;
}

// n tokens, or n values of `size` bytes.
aspis_status check_array(const char *who, const char *name, const void *at, int64_t n, int size) {
    if (n > 0 && (at == nullptr || (uintptr_t)at % size != 0))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: %s is NULL or misaligned", who, name);
    return ASPIS_OK;
}

aspis_status check_tokens(const char *who, const void *tokens, int64_t n, int index) {
    if (index != ASPIS_I32 && index != ASPIS_I64)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown token type %d", who, index);
    return check_array(who, "tokens", tokens, n, index == ASPIS_I64 ? 8 : 4);
}

aspis_status check_workspace(const char *who, const void *ws, size_t have, size_t need) {
    if (need > 0 && (ws == nullptr || have < need))
        return fail(ASPIS_ERR_BUFFER_SMALL, "%s: workspace of %zu bytes, %zu needed", who,
                    ws == nullptr ? (size_t)0 : have, need);
    if ((uintptr_t)ws % 16 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", who);
    return ASPIS_OK;
}

#define CHECK(call)                              \
    do {                                         \
        const aspis_status st_ = (call);         \
        if (st_ != ASPIS_OK) return st_;         \
    } while (0)

}  // namespace

extern "C" {

aspis_status aspis_embed(const void *table, int64_t vocab, int64_t d, int64_t ld,
                         aspis_dtype dtype, const void *tokens, int64_t n, aspis_index index,
                         double scale, void *out, int64_t ldo, aspis_dtype out_dtype,
                         void *stream) {
    const char *who = "aspis_embed";
    const Rows from{"table", table, vocab, d, ld, dtype}, to{"out", out, n, d, ldo, out_dtype};
    CHECK(check_rows(who, from));
    CHECK(check_rows(who, to));
    if (vocab > aspis::kMaxVocab)
        return fail(ASPIS_ERR_OVERFLOW, "%s: vocab=%lld", who, (long long)vocab);
    CHECK(check_tokens(who, tokens, n, index));
    if (!std::isfinite((float)scale))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: scale=%g", who, scale);
    CHECK(check_apart(who, {to}, {from, array("tokens", tokens, n, index == ASPIS_I64 ? 8 : 4)}));
    const aspis::EmbedArgs a{table, vocab, d, ld, dtype, {tokens, index == ASPIS_I64}, n,
                             (float)scale, out, ldo, out_dtype};
    return launched(aspis::launch_embed(a, static_cast<hipStream_t>(stream)), who);
}

size_t aspis_embed_workspace(int64_t n, int64_t d) {
    if (n < 0 || n > aspis::kMaxTokens || d < 0 || d > kMaxElements / (n < 1 ? 1 : n) / 16)
        return SIZE_MAX;
    return aspis::embed_grad_plan(n, d).bytes;
}

aspis_status aspis_embed_grad(const void *grad, int64_t n, int64_t d, int64_t ld,
                              aspis_dtype dtype, const void *tokens, aspis_index index,
                              double scale, void *out, int64_t vocab, int64_t ldo,
                              aspis_dtype out_dtype, uint32_t flags, void *workspace,
                              size_t ws_bytes, void *stream) {
    const char *who = "aspis_embed_grad";
    const Rows from{"grad", grad, n, d, ld, dtype}, to{"out", out, vocab, d, ldo, out_dtype};
    CHECK(check_rows(who, from));
    CHECK(check_rows(who, to));
    const size_t need = aspis_embed_workspace(n, d);
    if (vocab > aspis::kMaxVocab || need == SIZE_MAX)
        return fail(ASPIS_ERR_OVERFLOW, "%s: n=%lld d=%lld vocab=%lld", who, (long long)n,
                    (long long)d, (long long)vocab);
    CHECK(check_tokens(who, tokens, n, index));
    if (!std::isfinite((float)scale))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: scale=%g", who, scale);
    if (flags & ~ASPIS_EMBED_ACCUMULATE)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: unknown flags 0x%x", who, flags);
    CHECK(check_workspace(who, workspace, ws_bytes, need));
    CHECK(check_apart(who, {to, array("workspace", workspace, need, 1)},
                      {from, array("tokens", tokens, n, index == ASPIS_I64 ? 8 : 4)}));
    const aspis::EmbedGradArgs a{grad, n, d, ld, dtype, {tokens, index == ASPIS_I64},
                                 (float)scale, out, vocab, ldo, out_dtype,
                                 (flags & ASPIS_EMBED_ACCUMULATE) != 0, workspace};
    return launched(aspis::launch_embed_grad(a, static_cast<hipStream_t>(stream)), who);
}

aspis_status aspis_dropout(const void *x, int64_t rows, int64_t d, int64_t ld,
                           aspis_dtype dtype, double p, uint64_t seed, const uint64_t *seed_at,
                           uint64_t offset, const void *residual, int64_t ldr, void *out,
                           int64_t ldo, void *stream) {
    const char *who = "aspis_dropout";
    const Rows from{"x", x, rows, d, ld, dtype}, to{"out", out, rows, d, ldo, dtype};
    const Rows res{"residual", residual, rows, d, ldr, dtype};
    CHECK(check_rows(who, from));
    CHECK(check_rows(who, to));
    if (residual != nullptr) CHECK(check_rows(who, res));
    if (!(p >= 0.0 && p <= 1.0)) return fail(ASPIS_ERR_INVALID_ARG, "%s: p=%g", who, p);
    if ((uintptr_t)seed_at % 8 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: seed_at is misaligned", who);
    if ((!same(from, to) && overlap(from, to)) ||
        (residual != nullptr && !same(res, to) && overlap(res, to)))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: out overlaps an input without being it", who);
    CHECK(check_apart(who, {to}, {array("seed_at", seed_at, 1, 8)}));
    const double limit = std::nearbyint(p * 65536.0);
    const aspis::DropoutArgs a{x, rows, d, ld, dtype, (uint32_t)limit,
                               limit < 65536.0 ? (float)(65536.0 / (65536.0 - limit)) : 0.0f, seed,
                               seed_at, offset, residual, ldr, out, ldo};
    return launched(aspis::launch_dropout(a, static_cast<hipStream_t>(stream)), who);
}

size_t aspis_policy_workspace(int64_t rows, int64_t vocab, aspis_dtype dtype) {
    if (elem_bytes(dtype) == 0 || rows < 0 || rows > aspis::kMaxTokens || vocab < 0 ||
        vocab > aspis::kMaxLogits)
        return SIZE_MAX;
    return aspis::policy_plan(rows, vocab, elem_bytes(dtype)).bytes;
}

namespace {

// What the two calls on logits check alike.  need: bytes of workspace.
aspis_status check_logits(const char *who, const Rows &z, const void *tokens, int index,
                          double temperature, const float *logps, const void *ws,
                          size_t ws_bytes, size_t &need) {
    CHECK(check_rows(who, z));
    need = aspis_policy_workspace(z.rows, z.d, (aspis_dtype)z.dtype);
    if (need == SIZE_MAX)
        return fail(ASPIS_ERR_OVERFLOW, "%s: rows=%lld vocab=%lld", who, (long long)z.rows,
                    (long long)z.d);
    CHECK(check_tokens(who, tokens, z.rows, index));
    CHECK(check_array(who, "logps", logps, z.rows, 4));
    // (a temperature whose inverse or logarithms leave f32 is none)
    if (!(temperature >= 1e-30 && temperature <= 1e30))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: temperature=%g", who, temperature);
    return check_workspace(who, ws, ws_bytes, need);
}

}  // namespace

aspis_status aspis_token_logps(const void *logits, int64_t rows, int64_t vocab, int64_t ld,
                               aspis_dtype dtype, const void *tokens, aspis_index index,
                               double temperature, float *logps, void *workspace,
                               size_t ws_bytes, void *stream) {
    const char *who = "aspis_token_logps";
    const Rows z{"logits", logits, rows, vocab, ld, dtype};
    size_t need;
    CHECK(check_logits(who, z, tokens, index, temperature, logps, workspace, ws_bytes, need));
    CHECK(check_apart(who, {array("logps", logps, rows, 4), array("workspace", workspace, need, 1)},
                      {z, array("tokens", tokens, rows, index == ASPIS_I64 ? 8 : 4)}));
    aspis::PolicyArgs a{};
    a.logits = logits;
    a.rows = rows;
    a.vocab = vocab;
    a.ld = ld;
    a.dtype = dtype;
    a.tokens = {tokens, index == ASPIS_I64};
    a.inv_temperature = 1.0 / temperature;
    a.logps = logps;
    a.ws = workspace;
    return launched(aspis::launch_policy(a, static_cast<hipStream_t>(stream)), who);
}

aspis_status aspis_policy_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld,
                               aspis_dtype dtype, const void *tokens, aspis_index index,
                               const float *old, const float *advantage, const float *weight,
                               const float *ref, const aspis_policy *opt, float *sums,
                               float *logps, void *grad, int64_t ldg, void *workspace,
                               size_t ws_bytes, void *stream) {
    const char *who = "aspis_policy_loss";
    if (opt == nullptr) return fail(ASPIS_ERR_INVALID_ARG, "%s: NULL options", who);
    const Rows z{"logits", logits, rows, vocab, ld, dtype};
    const Rows g{"grad", grad, rows, vocab, ldg, dtype};
    size_t need;
    CHECK(check_logits(who, z, tokens, index, opt->temperature, logps, workspace, ws_bytes, need));
    CHECK(check_array(who, "old", old, rows, 4));
    CHECK(check_array(who, "advantage", advantage, rows, 4));
    CHECK(check_array(who, "weight", weight, rows, 4));
    CHECK(check_array(who, "sums", sums, 1, 4));
    if ((uintptr_t)ref % 4 != 0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: ref is misaligned", who);
    if (grad != nullptr) {
        CHECK(check_rows(who, g));
        if (!same(z, g) && overlap(z, g))
            return fail(ASPIS_ERR_INVALID_ARG, "%s: grad overlaps the logits without being them",
                        who);
    }
    if (!(opt->clip_low >= 0.0 && opt->clip_low <= 1.0) ||
        !(opt->clip_high >= 0.0 && std::isfinite((float)(1.0 + opt->clip_high))) ||
        !(opt->kl >= 0.0 && std::isfinite((float)opt->kl)) ||
        !std::isfinite((float)(opt->grad_scale / opt->temperature)))
        return fail(ASPIS_ERR_INVALID_ARG, "%s: clip_low=%g clip_high=%g kl=%g grad_scale=%g", who,
                    opt->clip_low, opt->clip_high, opt->kl, opt->grad_scale);
    // a position's inputs are read by several waves, after one may have written
    const Rows to = grad != nullptr ? g : Rows{"grad", nullptr, 0, 0, 0, dtype};
    CHECK(check_apart(who,
                      {to, array("logps", logps, rows, 4), array("sums", sums, 3, 4),
                       array("workspace", workspace, need, 1)},
                      {array("tokens", tokens, rows, index == ASPIS_I64 ? 8 : 4),
                       array("old", old, rows, 4), array("advantage", advantage, rows, 4),
                       array("weight", weight, rows, 4), array("ref", ref, rows, 4)}));
    CHECK(check_apart(who,
                      {array("logps", logps, rows, 4), array("sums", sums, 3, 4),
                       array("workspace", workspace, need, 1)}, {z}));
    if (rows > 0 && ref == nullptr && opt->kl != 0.0)
        return fail(ASPIS_ERR_INVALID_ARG, "%s: kl=%g without ref", who, opt->kl);
    const aspis::PolicyArgs a{logits, rows, vocab, ld, dtype, {tokens, index == ASPIS_I64},
                              1.0 / opt->temperature, old, advantage, weight, ref,
                              (float)(1.0 - opt->clip_low), (float)(1.0 + opt->clip_high),
                              (float)opt->kl, (float)(opt->grad_scale / opt->temperature), sums,
                              logps, grad, ldg, workspace};
    return launched(aspis::launch_policy(a, static_cast<hipStream_t>(stream)), who);
}

}  // extern "C"
