// Program for a host-only sanitizer build of the operators by which compressed models are judged and tuned: sizes, plans and
// the argument checks that reject a call before anything is launched.  Exit status 0 = clean.
#include <climits>
#include <cstdio>
#include <initializer_list>

#include "obc.h"

#define EXPECT(cond) do { if (!(cond)) { std::fprintf(stderr, "failed: %s\n", #cond); return 1; } } while (0)

int main()
{
    size_t n = 0;
    for (int T : {0, 1, 7, 511, 512, 513, 4096, 1 << 20, INT_MAX})
        for (int V : {1, 2, 1023, 32769, 131072, 1 << 20, 1 << 30}) {
            if ((long long)T * V > (1ll << 44)) continue;
            for (int type = OBC_F32; type <= OBC_BF16; ++type)
                for (int k : {0, 1, 255, 257, 1024}) EXPECT(obc_score_workspace_bytes(T, V, type, k, &n) == OBC_OK);
            for (int d : {1, 2048, 2049, 1 << 20}) {
                if ((long long)T * d > (1ll << 40)) continue;
                EXPECT(obc_embed_grad_workspace_bytes(T, V, d, &n) == OBC_OK && n >= (size_t)V * 8 + (size_t)T * 4);
                EXPECT(obc_layernorm_grad_workspace_bytes(T, d, &n) == OBC_OK);
            }
        }
    EXPECT(obc_score_workspace_bytes(1, 5, OBC_I8, 1, &n) == OBC_ERR_BAD_ARG);
    EXPECT(obc_score_workspace_bytes(1, 5, OBC_F32, 1025, &n) == OBC_ERR_BAD_ARG);
    EXPECT(obc_embed_grad_workspace_bytes(-1, 5, 5, &n) == OBC_ERR_BAD_ARG);
    EXPECT(obc_embed_grad_workspace_bytes(1, 5, 5, nullptr) == OBC_ERR_BAD_ARG);
    EXPECT(obc_layernorm_grad_workspace_bytes(-1, 4, &n) == OBC_ERR_BAD_ARG);
    for (int count : {0, 1, 63, 64, 65, 1000, INT_MAX}) EXPECT(obc_adamw_plan_bytes(count, &n) == OBC_OK);
    EXPECT(obc_adamw_plan_bytes(-1, &n) == OBC_ERR_BAD_ARG);
    // a null context is refused before anything else is looked at
    float f = 0.f;
    int32_t i = 0;
    int64_t w = 0;
    obc_adamw_tensor t = {};
    EXPECT(obc_score(nullptr, &f, OBC_F32, 1, 1, 1, &i, 1.f, 1, &f, &f, &f, &i, &f, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_layernorm(nullptr, &f, nullptr, OBC_F32, &f, &f, 0.f, 1, 1, nullptr, &f, OBC_F32, nullptr, nullptr, nullptr) == OBC_ERR_BAD_ARG);
    EXPECT(obc_layernorm_grad(nullptr, &f, &f, &f, &f, &f, nullptr, OBC_F32, 1, 1, &f, &f, &f, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_embed(nullptr, &f, OBC_F32, 1, 1, 1, &i, 1, 1.f, &f, OBC_F32, 1) == OBC_ERR_BAD_ARG);
    EXPECT(obc_embed_grad(nullptr, &i, 1, &f, OBC_F32, 1, 1.f, 1, 1, 0, &f, OBC_F32, 1, nullptr, 0) == OBC_ERR_BAD_ARG);
    EXPECT(obc_adamw_plan(nullptr, &t, 1, OBC_F32, 32, &f, &w) == OBC_ERR_BAD_ARG);
    EXPECT(obc_adamw(nullptr, &f, 1, 1, OBC_F32, 32, 1, nullptr, 0.1f, nullptr, 0.9, 0.999, 1e-8f, nullptr, 0) == OBC_ERR_BAD_ARG);
    std::puts("operators' host sanitizer run clean");
    return 0;
}
