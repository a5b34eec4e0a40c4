// Which tenants gacer_place_streams takes for the heavier ones, on a HIP runtime made of host code whose streams all run beside each other: the heaviest tenant
// comes first and takes queue 0.  Exit code 0 = every check held.
#include <hip/hip_runtime_api.h>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
#include "../../include/gacer.h"

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); std::exit(1); } } while (0)

extern "C" hipError_t __wrap_hipEventElapsedTime(float *ms, hipEvent_t, hipEvent_t) { *ms = 0.1f; return hipSuccess; }      // of two spins: one spin's time

static void *at(int i) { return (char *)0x10000 + ((size_t)i << 31); }      // aligned, never dereferenced

// a tenant of one operator over tensors [batch 1, features, rows, 1], its descriptor at an odd address
struct One {
    gacer_op op;
    std::vector<gacer_tensor> tensors;
    std::vector<char> desc;
    gacer_tenant t;
    One(gacer_opkind kind, int rows, int in, int out, gacer_dtype dtype, bool codes = false)
    {
        std::memset(&op, 0, sizeof op);
        std::memset(&t, 0, sizeof t);
        tensors = {{1, in, rows, 1, at(0)}, {1, out, rows, 1, at(1)}};
        op.kind = kind; op.in0 = op.in1 = op.res = -1; op.out = codes ? -1 : 1; op.kh = op.kw = op.stride = op.groups = 1; op.cin = in; op.cout = out;
        const gacer_fp8_rows x = {at(2), (float *)at(3), rows, in}, y = {at(4), (float *)at(5), rows, out}, none = {};
        const gacer_fp8_weight w = {at(6), (const float *)at(7)};
        const gacer_fp8_gemm g = {x, w};
        const gacer_fp8_gated f = {x, w, w, codes ? y : none};
        if (kind == GACER_GEMM) { op.in0 = 0; op.w = at(6); }
        else {
            const size_t n = kind == GACER_GATED_FP8 ? sizeof f : sizeof g;      // no byte more than the operator's own descriptor
            desc.resize(n + 1);
            std::memcpy(desc.data() + 1, kind == GACER_GATED_FP8 ? (const void *)&f : (const void *)&g, n);
            op.w = desc.data() + 1;
        }
        t.n_ops = 1; t.ops = &op; t.n_tensors = 2; t.tensors = tensors.data(); t.input = 0; t.output = 1; t.dtype = dtype; t.batch = 1;
    }
};

// the order in which the tenants take queues
static std::vector<int> queues(const std::vector<gacer_tenant> &tenants)
{
    void *streams[8];
    for (int i = 0; i < 8; ++i) streams[i] = at(20 + i);
    std::vector<int> chosen(tenants.size()), queue(tenants.size());
    int n = 0;
    CHECK(gacer_place_streams(tenants.data(), (int)tenants.size(), streams, 8, chosen.data(), queue.data(), &n, nullptr) == GACER_OK && n == 8);
    return queue;
}

int main()
{
    const std::vector<int> as_listed = {0, 1, 2}, turned = {2, 1, 0};
    One small(GACER_GEMM, 64, 512, 512, GACER_BF16), gemm(GACER_GEMM, 2048, 4096, 4096, GACER_BF16);
    One product(GACER_GEMM_FP8, 4096, 4096, 4096, GACER_BF16), block(GACER_GATED_FP8, 4096, 4096, 4096, GACER_BF16, true), kept(GACER_GATED_FP8, 4096, 4096, 4096, GACER_BF16);
    CHECK(queues({small.t, gemm.t, product.t}) == turned);       // a product of 8-bit rows is heavier than a plain one of half its size
    CHECK(queues({gemm.t, product.t, block.t}) == turned);       // a gated block has two products, whether it leaves codes
    CHECK(queues({gemm.t, product.t, kept.t}) == turned);        // or a tensor
    CHECK(queues({block.t, product.t, gemm.t}) == as_listed);
    One block32(GACER_GATED_FP8, 4096, 4096, 4096, GACER_F32, true), gemm32(GACER_GEMM, 4096, 4096, 4096, GACER_F32);
    CHECK(queues({block32.t, gemm32.t}) == (std::vector<int>{1, 0}));      // 8-bit products run at the rate of bf16 in a tenant of either type
    One bare(GACER_GATED_FP8, 64, 512, 512, GACER_BF16, true), lost(GACER_GEMM_FP8, 64, 512, 512, GACER_BF16);
    bare.op.w = nullptr;                                         // what gacer_load_tenants will refuse
    lost.op.out = 99;
    CHECK(queues({bare.t, lost.t, gemm.t}) == (std::vector<int>{1, 2, 0}));
    std::printf("all checks held\n");
    return 0;
}
