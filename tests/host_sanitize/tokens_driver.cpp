// tokens_driver.cpp -- the token operators' host code over random arguments,
// valid and not; the launchers are stubs that accept what reaches them.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../../include/aspis.h"
#include "../../paper_2108_02416_amd/csrc/aspis_tokens.h"

namespace aspis {
static int64_t reached = 0;
hipError_t launch_embed(const EmbedArgs &a, hipStream_t) {
    reached += a.n >= 0 && a.d >= 0 && a.ld >= a.d && a.ldo >= a.d;
    return hipSuccess;
}
hipError_t launch_embed_grad(const EmbedGradArgs &a, hipStream_t) {
    const EmbedGradPlan p = embed_grad_plan(a.n, a.d);
    if ((p.blocks << (p.shift + 1)) < a.n || p.words < (size_t)a.n * 4 + 32 || p.words % 16 != 0) abort();
    if (p.bytes != 4 * p.words + (size_t)p.blocks * 2 * embed_row(a.d) * 4) abort();
    ++reached;
    return hipSuccess;
}
hipError_t launch_dropout(const DropoutArgs &a, hipStream_t) {
    if (a.limit > 65536 || (a.limit < 65536 && !(a.scale >= 1.0f && a.scale <= 65536.0f))) abort();
    ++reached;
    return hipSuccess;
}
hipError_t launch_policy(const PolicyArgs &a, hipStream_t) {
    const PolicyPlan p = policy_plan(a.rows, a.vocab, a.dtype == ASPIS_F32 ? 4 : 2);
    if (p.units < 1 || p.stats % 8 != 0 || p.at % 4 != 0 || p.bytes % 16 != 0) abort();
    if (p.bytes < p.at + (size_t)a.rows * 4 || p.at != p.stats + (size_t)(a.rows * p.units) * 8)
        abort();
    ++reached;
    return hipSuccess;
}
}  // namespace aspis

int main() {
    std::mt19937_64 rng(5);
    auto pick = [&](std::initializer_list<int64_t> v) { return v.begin()[rng() % v.size()]; };
    auto size = [&]() {
        return pick({0, 1, 2, 7, 257, 2048, 70001, 1 << 24, -1, INT64_MAX, INT64_MIN,
                     int64_t(1) << 31, int64_t(1) << 40, int64_t(1) << 60});
    };
    auto at = [&]() { return (void *)(uintptr_t)pick({0, 1 << 20, (1 << 20) + 2, 1 << 28, 1 << 21}); };
    auto real = [&]() {
        const double v[] = {0.0, 0.1, 1.0, 2.0, -1.0, 1e300, 1e-40, INFINITY, NAN, 0.5, 1e-31};
        return v[rng() % 11];
    };
    int64_t ok = 0, refused = 0;
    for (int i = 0; i < 400000; ++i) {
        const int64_t n = size(), d = size(), v = size();
        const int64_t ld = rng() % 3 ? d : size(), ldo = rng() % 3 ? d : size();
        const aspis_dtype t = (aspis_dtype)(rng() % 20 == 0 ? 3 : rng() % 3);
        const aspis_index x = (aspis_index)(rng() % 2);
        const size_t room = rng() % 3 ? SIZE_MAX : (size_t)size();
        aspis_status st;
        switch (i % 5) {
            case 0: st = aspis_embed(at(), v, d, ld, t, at(), n, x, real(), at(), ldo, t, nullptr); break;
            case 1:
                st = aspis_embed_grad(at(), n, d, ld, t, at(), x, real(), at(), v, ldo, t,
                                      (uint32_t)(rng() % 3), at(), room, nullptr);
                break;
            case 2:
                st = aspis_dropout(at(), n, d, ld, t, real(), rng(), (const uint64_t *)at(), rng(), at(),
                                   ld, at(), ldo, nullptr);
                break;
            case 3:
                st = aspis_token_logps(at(), n, d, ld, t, at(), x, real(), (float *)at(), at(), room,
                                       nullptr);
                break;
            default: {
                const aspis_policy o{real(), real(), real(), real(), real()};
                st = aspis_policy_loss(at(), n, d, ld, t, at(), x, (float *)at(), (float *)at(),
                                       (float *)at(), (float *)at(), &o, (float *)at(), (float *)at(),
                                       at(), ldo, at(), room, nullptr);
            }
        }
        if (st == ASPIS_OK) ++ok;
        else ++refused;
    }
    if (ok != aspis::reached || ok < 1000 || refused < 100000) {
        printf("ok %lld reached %lld refused %lld\n", (long long)ok, (long long)aspis::reached,
               (long long)refused);
        return 1;
    }
    printf("ok\n");
    return 0;
}
