// Program for a host-only sanitizer build of the operators around compressed layers: sizes, plans and the argument
// checks that reject a call before anything is launched.  Exit status 0 = clean.
#include <climits>
#include <cstdio>
#include <initializer_list>

#include "obc.h"

#define EXPECT(cond) do { if (!(cond)) { std::fprintf(stderr, "failed: %s\n", #cond); return 1; } } while (0)

int main()
{
    size_t n = 0;
    for (int R : {0, 1, 16, 17, 768, 16384, INT_MAX})
        for (int d : {1, 31, 128, 129, 4096, 65536, INT_MAX})
            for (int group : {0, 32, 64, 128, 256, 384, INT_MAX}) {
                if ((long long)R * d > (1ll << 40)) continue;
                int rc = obc_pack4_bytes(R, d, group, &n);
                EXPECT(rc == OBC_OK || (rc == OBC_ERR_BAD_ARG && group == INT_MAX && group < d));
                for (int T : {0, 1, 16, 17, 32, 33, 64, 65, 5000}) {
                    if ((long long)T * R > (1ll << 36) || (long long)T * d > (1ll << 36) || R == INT_MAX || d == INT_MAX) continue;
                    for (int type = OBC_F32; type <= OBC_I8; ++type) {
                        EXPECT(obc_product4_workspace_bytes(T, R, d, group, type, &n) == OBC_OK);
                        rc = obc_product4_grad_workspace_bytes(T, R, d, group, type, &n);
                        EXPECT(rc == (type == OBC_I8 ? OBC_ERR_BAD_ARG : OBC_OK));
                    }
                }
            }
    for (int group : {-1, 1, 48, 130}) EXPECT(obc_pack4_bytes(4, 1000, group, &n) == OBC_ERR_BAD_ARG);
    EXPECT(obc_pack4_bytes(4, 4, 0, nullptr) == OBC_ERR_BAD_ARG);
    EXPECT(obc_rmsnorm_grad_workspace_bytes(4096, 65536, &n) == OBC_OK && n >= (size_t)65536 * 4);
    EXPECT(obc_rmsnorm_grad_workspace_bytes(-1, 4, &n) == OBC_ERR_BAD_ARG);
    // a null context is refused before anything else is looked at
    float f = 0.f;
    int32_t i = 0;
    EXPECT(obc_group_grid(nullptr, &f, nullptr, 1, 1, 0, 15, 0, &f, &f) == OBC_ERR_BAD_ARG);
    EXPECT(obc_pack4(nullptr, &i, &f, &f, 1, 1, 0, &f) == OBC_ERR_BAD_ARG);
    EXPECT(obc_product4(nullptr, &f, 1, 1, 0, &f, OBC_F32, nullptr, 1, 1, &f, OBC_F32, 1, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_product4_grad(nullptr, &f, 1, 1, 0, &f, OBC_F32, 1, 1, &f, 1, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_rmsnorm(nullptr, &f, nullptr, OBC_F32, &f, 0.f, 1, 1, nullptr, &f, OBC_F32, nullptr, nullptr) == OBC_ERR_BAD_ARG);
    EXPECT(obc_rmsnorm_grad(nullptr, &f, &f, &f, &f, nullptr, OBC_F32, 1, 1, &f, &f, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_distill(nullptr, &f, OBC_F32, 1, 1, 1, &i, &f, 1, 1.f, nullptr, &f, nullptr, 0) == OBC_ERR_BAD_ARG);
    std::puts("operators' host sanitizer run clean");
    return 0;
}
