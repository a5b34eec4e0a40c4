// Host-side exerciser of the C ABI with operators of a decoding tenant, for sanitizer builds: two of them have no output tensor and one has no
// input tensor, which every walk over a tenant's operators has to allow for.  Kernels are geometry-only, the HIP runtime is host code
// (stub_hip.cpp), so that rounds, profiles and traces are walked through as well.  Exit code 0 = every check held.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <string>
#include <vector>
#include "../../include/gacer.h"
#include "token_kernels.h"

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, ctx ? gacer_last_error(ctx) : ""); std::exit(1); } } while (0)

static void *const FAKE = (void *)0x10000;      // aligned, never dereferenced
static void *at(int i) { return (char *)FAKE + ((size_t)i << 28); }

// a step of a decoder: rotation (in place or not), write, attention, read back, product, sampling
struct Step {
    gacer_rope rope;
    gacer_cache cache;
    gacer_sampling sampling;
    std::vector<gacer_op> ops;
    std::vector<gacer_tensor> tensors;
    gacer_tenant desc;
    Step(int batch, int S, gacer_dtype dtype, bool in_place, int max_pages, std::mt19937 &rng)
    {
        const int kv = 1 + (int)(rng() % 3), heads = kv * (1 + (int)(rng() % 4)), dim = rng() % 2 ? 64 : 128, vocab = 1000 + (int)(rng() % 100);
        rope = {heads, kv, dim, dim, (int)(rng() % 2), 1, {dim / 2, 0, 0}, 100, (const float *)FAKE, (const int *)FAKE};
        if (rng() % 4 == 0) rope.rotary_dims = 0, rope.n_axes = (int)rng(), rope.sections[1] = (int)rng();      // norms alone: the rotation's fields may hold anything
        cache = {heads, kv, dim, 64, 10, max_pages, (int)(rng() % 2) * 100, FAKE, FAKE, (unsigned *)FAKE, (unsigned *)FAKE, (const int *)FAKE, (const int *)FAKE, nullptr};
        sampling = {(const float *)FAKE, nullptr, nullptr, nullptr, nullptr, (int *)FAKE, nullptr};
        const int64_t w = (int64_t)(heads + 2 * kv) * dim;
        tensors = {{batch, w, S, 1, at(1)}, {batch, w, S, 1, in_place ? at(1) : at(2)}, {batch, heads * dim, S, 1, at(3)},
                   {batch, 2 * kv * dim, S, 1, at(4)}, {batch, vocab, S, 1, at(5)}};
        auto op = [&](gacer_opkind kind, int in0, int out, const void *w_) {
            gacer_op o;
            std::memset(&o, 0, sizeof o);
            o.kind = kind; o.in0 = in0; o.in1 = o.res = -1; o.out = out; o.w = w_; o.kh = o.kw = o.stride = o.groups = 1; o.alpha = 0.125f;
            ops.push_back(o);
        };
        op(GACER_QKNORM_ROPE, 0, 1, &rope);
        op(GACER_CACHE_WRITE, 1, -1, &cache);
        op(GACER_CACHE_ATTENTION, 1, 2, &cache);
        op(GACER_CACHE_READ, -1, 3, &cache);
        op(GACER_GEMM, 2, 4, FAKE);
        ops.back().cin = heads * dim; ops.back().cout = vocab;
        op(GACER_SAMPLE, 4, -1, &sampling);
        std::memset(&desc, 0, sizeof desc);
        desc.n_ops = (int)ops.size(); desc.ops = ops.data(); desc.n_tensors = (int)tensors.size(); desc.tensors = tensors.data();
        desc.input = 0; desc.output = 4; desc.dtype = dtype; desc.batch = batch;
    }
};

int main()
{
    std::mt19937 rng(5);
    for (int trial = 0; trial < 24; ++trial) {
        gacer_ctx *ctx = nullptr;
        gacer::current_device = trial % 2;
        CHECK(gacer_create(&ctx) == GACER_OK);
        const bool in_place = trial % 2, two = trial % 3 == 0;
        const int batch = 1 + (int)(rng() % 9);
        std::vector<Step> steps;
        steps.reserve(2);
        for (int t = 0; t < 1 + two; ++t) steps.emplace_back(batch, 1 + (int)(rng() % 40), trial % 4 < 2 ? GACER_F32 : GACER_BF16, in_place, trial % 5 ? 3 : 2000, rng);
        std::vector<gacer_tenant> descs;
        for (Step &s : steps) {
            s.desc.ops = s.ops.data(); s.desc.tensors = s.tensors.data();
            s.ops[0].w = &s.rope; s.ops[1].w = s.ops[2].w = s.ops[3].w = &s.cache; s.ops[5].w = &s.sampling;
            s.desc.stream = two ? at(20 + (int)descs.size()) : nullptr;
            descs.push_back(s.desc);
        }
        const int NT = (int)descs.size(), n_ops = (int)steps[0].ops.size();
        CHECK(gacer_load_tenants(ctx, descs.data(), NT) == GACER_OK);
        int count = 0;
        CHECK(gacer_launch_count(ctx, GACER_MODE_SEQUENTIAL, &count) == GACER_OK && count == NT * n_ops);
        // refusals, field by field, leave what is loaded usable
        for (int k = 0; k < 40; ++k) {
            Step bad = steps[0];
            bad.desc.ops = bad.ops.data(); bad.desc.tensors = bad.tensors.data();
            int *const fields = k % 2 ? &bad.rope.heads : &bad.cache.heads;
            fields[rng() % 7] = (int)rng();
            bad.ops[0].w = &bad.rope; bad.ops[1].w = bad.ops[2].w = bad.ops[3].w = &bad.cache;
            (k % 3 ? bad.ops[rng() % n_ops].in0 : bad.ops[rng() % n_ops].out) = (int)(rng() % 9) - 2;
            gacer_ctx *other = nullptr;
            CHECK(gacer_create(&other) == GACER_OK);
            (void)gacer_load_tenants(other, &bad.desc, 1);
            gacer_destroy(other);
        }
        {   // a descriptor may stand at any address
            Step odd = steps[0];
            odd.desc.ops = odd.ops.data(); odd.desc.tensors = odd.tensors.data();
            std::vector<char> bytes[3] = {std::vector<char>(sizeof odd.rope + 1), std::vector<char>(sizeof odd.cache + 1), std::vector<char>(sizeof odd.sampling + 1)};
            std::memcpy(bytes[0].data() + 1, &odd.rope, sizeof odd.rope);
            std::memcpy(bytes[1].data() + 1, &odd.cache, sizeof odd.cache);
            std::memcpy(bytes[2].data() + 1, &odd.sampling, sizeof odd.sampling);
            odd.ops[0].w = bytes[0].data() + 1; odd.ops[1].w = odd.ops[2].w = odd.ops[3].w = bytes[1].data() + 1; odd.ops[5].w = bytes[2].data() + 1;
            gacer_ctx *other = nullptr;
            CHECK(gacer_create(&other) == GACER_OK);
            CHECK(gacer_load_tenants(other, &odd.desc, 1) == GACER_OK);
            gacer_destroy(other);
        }
        // every operator in two along the batch; none of them along its channels
        std::vector<gacer_split> sp;
        for (int i = 0; i < n_ops && batch >= 2; ++i) sp.push_back({0, i, GACER_AXIS_BATCH, 2, nullptr, 0});
        gacer_plan plan = {(int)sp.size(), sp.data(), 0, nullptr};
        CHECK(gacer_set_plan(ctx, &plan) == GACER_OK);
        for (int i : {0, 1, 2, 3, 5}) {
            gacer_split one = {0, i, GACER_AXIS_COUT, 2, nullptr, 0};
            gacer_plan wrong = {1, &one, 0, nullptr};
            CHECK(gacer_set_plan(ctx, &wrong) == GACER_EPLAN);
        }
        CHECK(gacer_set_plan(ctx, &plan) == GACER_OK);
        for (int mode : {GACER_MODE_PLAN, GACER_MODE_SEQUENTIAL, GACER_MODE_STREAM_PARALLEL}) {
            CHECK(gacer_run(ctx, mode, 2, nullptr) == GACER_OK);
            CHECK(gacer_run_static(ctx, mode, 1) == GACER_OK);
            size_t rows = 0;
            CHECK(gacer_trace_run(ctx, mode, 1, nullptr, 0, &rows) == GACER_OK && rows >= (size_t)(NT * n_ops));
            std::vector<gacer_launch_stat> stats(rows);
            CHECK(gacer_trace_run(ctx, mode, 1, stats.data(), rows, &rows) == GACER_OK);
        }
        for (int t = 0; t < NT; ++t) {
            const long before = gacer::token_launches.all;
            CHECK(gacer_enqueue(ctx, t, nullptr) == GACER_OK && gacer::token_launches.all == before + 5);
            const int own = gacer::current_device, other = 1 - own;          // on the context's GPU while another one is current
            gacer::current_device = other;
            CHECK(gacer_enqueue(ctx, t, nullptr) == GACER_OK && gacer::token_launches.device == own && gacer::current_device == other);
            gacer::current_device = own;
        }
        // the profile's own table, then random ones, with rows for axes that these operators do not have
        size_t n = 0;
        CHECK(gacer_profile(ctx, nullptr, 0, &n) == GACER_OK);
        std::vector<gacer_prof> table(n);
        const long own_before = gacer::token_launches.in_place_at[at(1)];
        CHECK(gacer_profile(ctx, table.data(), n, &n) == GACER_OK);
        // timed on other memory than the tenant's: on its own only in the rounds (one first, one more where a switch is timed)
        CHECK(gacer::token_launches.in_place_at[at(1)] - own_before == (in_place ? (two ? 4 : 1) : 0));
        for (int k = 0; k < 6; ++k) {
            std::vector<gacer_prof> prof;
            std::uniform_real_distribution<float> uT(0.1f, 2.0f), uW(0.05f, 1.0f);
            for (int t = 0; t < NT; ++t)
                for (int i = 0; i < n_ops; ++i) {
                    const float T = uT(rng), W = uW(rng);
                    prof.push_back({t, i, GACER_AXIS_NONE, 1, T, 10, W, 0.f});
                    for (int f = 2; f <= 8 && f <= batch; f *= 2) prof.push_back({t, i, GACER_AXIS_BATCH, f, T / f * 1.1f, 10, W / f, 0.f});
                }
            prof.push_back({-1, -1, GACER_AXIS_NONE, 1, 0.03f, 0, 1.f, 0.f});
            const std::vector<gacer_prof> &use = k ? prof : table;
            gacer_plan *found = nullptr;
            std::vector<int> ptrs(8 * NT);
            int n_ptr = 0;
            double R = 0, R2 = 0, makespan = 0;
            CHECK(gacer_search(ctx, use.data(), use.size(), 10, &found, ptrs.data(), &n_ptr, &R) == GACER_OK);
            for (int i = 0; i < found->n_split; ++i)
                CHECK(found->split[i].axis != GACER_AXIS_COUT || steps[found->split[i].tenant].ops[found->split[i].op].kind == GACER_GEMM);
            CHECK(gacer_set_plan(ctx, found) == GACER_OK);
            CHECK(gacer_model_residue(ctx, use.data(), use.size(), found->split, found->n_split, ptrs.data(), n_ptr, &R2, &makespan) == GACER_OK);
            gacer_plan *better = nullptr;
            float ms = 0.f;
            if (k == 1) {
                CHECK(gacer_refine(ctx, use.data(), use.size(), 2, 0.01f, &better, &ms) == GACER_OK);
                gacer_plan_free(better);
            }
            gacer_plan_free(found);
            for (int i : {0, 1, 2, 3, 5}) {
                std::vector<gacer_prof> bad = prof;
                bad.push_back({0, i, GACER_AXIS_COUT, 2, 0.01f, 10, 0.1f, 0.f});
                found = nullptr;
                CHECK(gacer_search(ctx, bad.data(), bad.size(), 10, &found, ptrs.data(), &n_ptr, &R) == GACER_EINVAL && !found);
            }
        }
        gacer_destroy(ctx);
    }
    gacer_ctx *ctx = nullptr;
    CHECK(gacer::token_launches.stray_positions == 0);
    std::printf("token driver: all checks held\n");
    return 0;
}
