// Program for a host-only sanitizer build of AdamW's plan: arrays that a step must not share.  Addresses are never followed; without a device, what
// is not refused fails at its launch.  Exit status 0 = clean.
#include <cstdio>

#include "../../paper_2208_11580_amd/csrc/common.h"

#define EXPECT(cond) do { if (!(cond)) { std::fprintf(stderr, "failed (line %d): %s\n", __LINE__, #cond); return 1; } } while (0)

namespace {

constexpr int64_t N = 1000;

void *at(uintptr_t a) { return (void *)a; }

// Tensor `i` in place, every array 1 MB from the next
obc_adamw_tensor tensor(int i, int bits, bool master)
{
    const uintptr_t base = (uintptr_t)(i + 1) << 28;
    obc_adamw_tensor t = {};
    t.n = N;
    t.p = t.p_out = at(base);
    t.g = at(base + (1 << 20));
    t.m = t.m_out = at(base + (2 << 20));
    t.v = t.v_out = at(base + (3 << 20));
    if (bits == 8) {
        t.m_scale = t.m_scale_out = (float *)at(base + (4 << 20));
        t.v_scale = t.v_scale_out = (float *)at(base + (5 << 20));
    }
    if (master) t.master = t.master_out = (float *)at(base + (6 << 20));
    return t;
}

int plan(const obc_adamw_tensor *t, int count, int type, int bits)
{
    obc_ctx ctx{};
    int64_t groups = 0;
    return obc_adamw_plan(&ctx, t, count, type, bits, at((uintptr_t)1 << 40), &groups);
}

}  // namespace

int main()
{
    for (int bits : {32, 8})
        for (int type : {OBC_F32, OBC_BF16})
            for (bool master : {false, true}) {
                const int e = type == OBC_F32 ? 4 : 2;
                obc_adamw_tensor t[3], u[3];
                for (int i = 0; i < 3; ++i) t[i] = tensor(i, bits, master);
                const auto refused = [&](auto change) {
                    for (int i = 0; i < 3; ++i) u[i] = t[i];
                    change();
                    return plan(u, 3, type, bits) == OBC_ERR_BAD_ARG;
                };
                // taken: in place; gradients that are shared, or the parameter itself; neighbours; empty tensors anywhere
                EXPECT(!refused([] {}));
                EXPECT(!refused([&] { u[1].g = u[0].g; }));
                EXPECT(!refused([&] { u[1].g = (char *)u[0].g + e; }));
                EXPECT(!refused([&] { u[1].g = u[1].p; }));
                EXPECT(!refused([&] { u[1].p_out = at((uintptr_t)u[1].g); }));
                EXPECT(!refused([&] { u[1].p = u[1].p_out = (char *)u[0].p + N * e; }));
                EXPECT(!refused([&] { u[1].g = (char *)u[0].p + N * e; }));
                EXPECT(!refused([&] { u[1].g = (char *)u[0].p - N * e; }));
                EXPECT(!refused([&] { u[1].p = u[1].p_out = (void *)u[0].p; u[1].n = 0; }));
                // outputs that overlap: a tensor listed twice, moments in each other's place, the last element
                EXPECT(refused([&] { u[1].p = u[1].p_out = (void *)u[0].p; }));
                EXPECT(refused([&] { u[2].m_out = u[0].m_out; }));
                EXPECT(refused([&] { u[2].p_out = (char *)u[0].v_out + N * (bits / 8) - 1 * e; }));
                // an output over another tensor's input: parameters that change places, moments, gradients
                EXPECT(refused([&] { u[0].p_out = (void *)u[1].p; u[1].p_out = (void *)u[0].p; }));
                EXPECT(refused([&] { u[0].p_out = (void *)u[1].p; u[1].p_out = at((uintptr_t)9 << 30); }));
                EXPECT(refused([&] { u[0].p_out = (void *)u[2].g; }));
                EXPECT(refused([&] { u[0].m_out = (void *)u[1].m; u[1].m_out = at((uintptr_t)9 << 30); }));
                EXPECT(refused([&] { u[2].g = u[0].p; }));
                // an output over an input of its own tensor, but not element for element
                EXPECT(refused([&] { u[1].p_out = (char *)u[1].p + e; }));
                EXPECT(refused([&] { u[1].p_out = (char *)u[1].g + 8 * e; }));
                EXPECT(refused([&] { u[1].p_out = (char *)u[1].g - (N - 1) * e; }));
                EXPECT(refused([&] { u[1].v_out = (char *)u[1].v + 4; }));
                if (bits / 8 != e) EXPECT(refused([&] { u[1].m_out = (void *)u[1].g; }));
                if (master) EXPECT(refused([&] { u[1].master_out = (float *)u[1].master + 1; }));
                if (master) EXPECT(refused([&] { u[0].master_out = (float *)u[1].master; u[1].master_out = (float *)at((uintptr_t)9 << 30); }));
                if (bits == 8) EXPECT(refused([&] { u[0].m_scale_out = (float *)u[1].m_scale; u[1].m_scale_out = (float *)at((uintptr_t)9 << 30); }));
            }
    std::puts("plan's host sanitizer run clean");
    return 0;
}
