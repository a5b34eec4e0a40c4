// Host-side exerciser of the C ABI with operators on 8-bit rows, for sanitizer builds: products have no input tensor, a gated block neither input nor output, and
// descriptors lie at odd addresses.  Kernels are geometry-only, the HIP runtime is host code (stub_hip.cpp).  Exit code 0 = every check held.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>
#include "../../include/gacer.h"
#include "token_kernels.h"

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, ctx ? gacer_last_error(ctx) : ""); std::exit(1); } } while (0)

static void *at(int i) { return (char *)0x10000 + ((size_t)i << 31); }      // aligned, never dereferenced

// the dense half of a layer: norm, product, codes, product with residual, norm with residual, gated block, product with residual, norm in the tenant's type
struct Layer {
    std::vector<char> descs;
    std::vector<gacer_op> ops;
    std::vector<gacer_tensor> tensors;
    gacer_tenant desc;
    int place = 20;
    gacer_fp8_rows rows(int n, int features) { place += 2; return {at(place), (float *)at(place + 1), n, features}; }
    gacer_fp8_weight weight() { place += 2; return {at(place), (const float *)at(place + 1)}; }
    template <typename D> void add(gacer_opkind kind, const D &d, int in0, int res, int out, gacer_act act = GACER_ACT_NONE)
    {
        gacer_op o;
        std::memset(&o, 0, sizeof o);
        o.kind = kind; o.in0 = in0; o.in1 = -1; o.res = res; o.out = out; o.kh = o.kw = o.stride = o.groups = 1; o.act = act; o.alpha = 1e-6f;
        o.w = (const void *)(uintptr_t)descs.size();
        descs.insert(descs.end(), (const char *)&d, (const char *)&d + sizeof d);
        descs.push_back(0);                                  // the next one lies at another alignment
        ops.push_back(o);
    }
    Layer(int batch, int S, gacer_dtype dtype, std::mt19937 &rng)
    {
        const int n = batch * S, w = 16 * (1 + (int)(rng() % 40)), q = 16 * (1 + (int)(rng() % 40)), f = 16 * (1 + (int)(rng() % 600)), odd = 1 + (int)(rng() % 5000);
        auto t = [&](int c) { tensors.push_back({batch, c, S, 1, at((int)tensors.size())}); return (int)tensors.size() - 1; };
        const int x = t(w), qkv = t(q), y = t(w), h = t(w), z = t(w), last = t(w), wide = t(odd);
        const gacer_fp8_rows n1 = rows(n, w), c1 = rows(n, q), n2 = rows(n, w), g1 = rows(n, f);
        descs.push_back(0);
        add(GACER_RMSNORM_FP8, gacer_fp8_norm{1, n1}, x, -1, -1);
        add(GACER_GEMM_FP8, gacer_fp8_gemm{n1, weight()}, -1, -1, qkv);
        add(GACER_RMSNORM_FP8, gacer_fp8_norm{0, c1}, qkv, -1, -1);
        add(GACER_GEMM_FP8, gacer_fp8_gemm{c1, weight()}, -1, -1, y);
        add(GACER_RMSNORM_FP8, gacer_fp8_norm{1, n2}, y, x, h);
        add(GACER_GATED_FP8, gacer_fp8_gated{n2, weight(), weight(), g1}, -1, -1, -1, GACER_ACT_SILU);
        add(GACER_GEMM_FP8, gacer_fp8_gemm{g1, weight()}, -1, h, z);
        add(GACER_RMSNORM_FP8, gacer_fp8_norm{1, gacer_fp8_rows{}}, z, -1, last);
        add(GACER_GATED_FP8, gacer_fp8_gated{n2, weight(), weight(), gacer_fp8_rows{}}, -1, -1, wide, GACER_ACT_GELU_TANH);
        for (gacer_op &o : ops) o.w = descs.data() + (uintptr_t)o.w;
        std::memset(&desc, 0, sizeof desc);
        desc.n_ops = (int)ops.size(); desc.ops = ops.data(); desc.n_tensors = (int)tensors.size(); desc.tensors = tensors.data();
        desc.input = x; desc.output = last; desc.dtype = dtype; desc.batch = batch;
    }
};

int main()
{
    std::mt19937 rng(7);
    for (int trial = 0; trial < 24; ++trial) {
        gacer_ctx *ctx = nullptr;
        CHECK(gacer_create(&ctx) == GACER_OK);
        const int batch = 1 + (int)(rng() % 6);
        Layer a(batch, 1 + (int)(rng() % 50), GACER_F32, rng), b(batch, 1, GACER_BF16, rng);
        gacer_tenant both[2] = {a.desc, b.desc};
        CHECK(gacer_load_tenants(ctx, both, 2) == GACER_OK);
        for (int k = 0; k < 60; ++k) {                       // any word of any descriptor, any index: loaded or refused, never followed
            std::vector<char> spoilt = a.descs;
            const uint32_t word = k % 3 ? (uint32_t)rng() : (uint32_t)(rng() % 64) - 16;
            std::memcpy(spoilt.data() + rng() % (spoilt.size() - 4), &word, 4);
            std::vector<gacer_op> ops = a.ops;
            for (gacer_op &o : ops) o.w = spoilt.data() + ((const char *)o.w - a.descs.data());
            if (k % 2) (k % 4 == 1 ? ops[rng() % ops.size()].res : ops[rng() % ops.size()].out) = (int)(rng() % 12) - 2;
            gacer_tenant t = a.desc;
            t.ops = ops.data();
            gacer_ctx *other = nullptr;
            CHECK(gacer_create(&other) == GACER_OK);
            if (gacer_load_tenants(other, &t, 1) != GACER_OK) CHECK(std::strstr(gacer_last_error(other), "tenant 0"));
            gacer_destroy(other);
        }
        for (Layer *l : {&a, &b}) std::fill(l->descs.begin(), l->descs.end(), (char)0xEE);      // copied when they were loaded
        for (int mode = 0; mode < 3; ++mode) CHECK(gacer_run(ctx, mode, 2, nullptr) == GACER_OK);
        CHECK(gacer_enqueue(ctx, 1, nullptr) == GACER_OK);
        size_t n = 0;
        CHECK(gacer_profile(ctx, nullptr, 0, &n) == GACER_OK);
        std::vector<gacer_prof> table(n);
        CHECK(gacer_profile(ctx, table.data(), n, &n) == GACER_OK);
        for (const gacer_prof &p : table) CHECK(p.axis != GACER_AXIS_COUT);
        gacer_plan *plan = nullptr;
        std::vector<int> P(2 * 64);
        int n_ptr = 0;
        double residue = 0;
        CHECK(gacer_search(ctx, table.data(), n, 20, &plan, P.data(), &n_ptr, &residue) == GACER_OK);
        CHECK(gacer_set_plan(ctx, plan) == GACER_OK);
        gacer_plan_free(plan);
        CHECK(gacer_run(ctx, GACER_MODE_PLAN, 1, nullptr) == GACER_OK);
        if (batch > 1) {
            std::vector<gacer_split> splits;
            for (int i = 0; i < (int)a.ops.size(); ++i) splits.push_back({0, i, GACER_AXIS_BATCH, 2, nullptr, 0});
            const gacer_plan cut = {(int)splits.size(), splits.data(), 0, nullptr};
            CHECK(gacer_set_plan(ctx, &cut) == GACER_OK && gacer_run(ctx, GACER_MODE_PLAN, 1, nullptr) == GACER_OK);
        }
        CHECK(gacer_trace_run(ctx, GACER_MODE_PLAN, 1, nullptr, 0, &n) == GACER_OK);
        std::vector<gacer_launch_stat> rows(n);
        CHECK(gacer_trace_run(ctx, GACER_MODE_PLAN, 1, rows.data(), n, &n) == GACER_OK);
        double flops = 0;
        for (const gacer_launch_stat &r : rows) { CHECK(r.bytes > 0); flops += r.flops; }
        CHECK(flops > 0);
        gacer_destroy(ctx);
    }
    std::printf("all checks held\n");
    return 0;
}
