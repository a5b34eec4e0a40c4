// What the launchers of the operators on 8-bit rows say of their kernels: one line for each kernel, its name as the compiler has it, workgroups a unit holds,
// LDS bytes, threads; and, with arguments "gated rows in out [codes]", the tile and slices that a product of that size takes (dry runs: nothing is launched, no GPU is needed).
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include <string>
#include "../paper_2304_11745_amd/csrc/kernels.h"
#include "../paper_2304_11745_amd/csrc/tokens_geom.h"

using namespace gacer;

static std::set<std::string> told;
static void tell(const std::string &name, const LaunchInfo &li)
{
    if (told.insert(name).second) std::printf("%s %d %d %d\n", name.c_str(), li.wg_per_cu, li.lds_bytes, li.threads);
}

static TokenArgs product(bool gated, int rows, int cin, int cout, bool codes, int dtype)
{
    TokenArgs a;
    std::memset(&a, 0, sizeof a);
    a.dtype = dtype; a.op = gated ? TK_GATED_FP8 : TK_GEMM_FP8; a.b_hi = a.batch = rows; a.S = 1; a.features = cout;
    a.xq = {(unsigned char *)0x10000, (float *)0x10000, rows, cin};      // aligned, never dereferenced
    a.w = a.w2 = {(const unsigned char *)0x10000, (const float *)0x10000};
    if (codes) a.yq = {(unsigned char *)0x10000, (float *)0x10000, rows, cout};
    else a.y = (void *)0x10000;
    return a;
}

int main(int argc, char **argv)
{
    if (argc > 4) {
        const TokenArgs a = product(std::atoi(argv[1]) != 0, std::atoi(argv[2]), std::atoi(argv[3]), std::atoi(argv[4]), argc > 5, DT_BF16);
        std::printf("%s %d\n", launch_gemm_fp8(a, nullptr, true, 1).kernel, fp8_geom(a).slices);
        return 0;
    }
    static const char *tiles[] = {"", "Li64ELi32E", "Li64ELi64E", "Li128ELi128E", "Li256ELi128E", "Li256ELi64E", "Li256ELi32E"};
    for (int dtype : {DT_F32, DT_BF16}) {
        const std::string type = dtype == DT_F32 ? "f" : "t";
        for (int gated : {0, 1})
            for (int rows : {1, 20, 40, 64, 128, 300, 512, 1024, 4096})
                for (int cin : {128, 1024, 3088, 8208, 14336})
                    for (int cout : {80, 512, 4096, 14336}) {
                        const TokenArgs a = product(gated, rows, cin, cout, gated, dtype);
                        const Fp8Geom g = fp8_geom(a);
                        const std::string name = g.tile == FP8_FEW ? "fp8_few_kernelI" + type + "E" : "fp8_tile_kernelI" + type + "Lb" + std::to_string(gated) + "E" + tiles[g.tile];
                        tell(name, launch_gemm_fp8(a, nullptr, true, 1));
                        if (g.slices > 1) tell("fp8_join_kernelI" + type + "Lb" + std::to_string(gated) + "ELi" + std::to_string(g.slices <= 2 ? 2 : g.slices <= 4 ? 4 : 8) + "E", launch_gemm_fp8(a, nullptr, true, 2));
                    }
        for (int runs : {128, 129, 1024, 1025, 2048, 4096, 8192, 1, 64, 65, 256, 257, 512})
            for (int odd : {0, 1}) {
                TokenArgs a;
                std::memset(&a, 0, sizeof a);
                a.dtype = dtype; a.op = TK_RMSNORM_FP8; a.b_hi = a.batch = 5; a.S = 1; a.features = runs * 8 - odd; a.x = a.y = (void *)0x10000;
                const int lanes = runs <= 128 ? 64 : runs <= 1024 ? 256 : 1024, each = (runs + lanes - 1) / lanes, r = each <= 1 ? 1 : each <= 2 || lanes == 1024 ? 2 : 4;
                tell("rmsnorm_fp8_kernelI" + type + "Li" + std::to_string(lanes) + "ELi" + std::to_string(r) + "ELb" + std::to_string(!odd) + "ELb" + std::to_string(lanes == 1024 && each > 2) + "E", launch_rmsnorm_fp8(a, nullptr, true));
            }
    }
    return 0;
}
