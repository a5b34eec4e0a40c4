// What the launchers of a decoding tenant's operators say of their kernels: one line for each kernel, its name as the compiler has it, workgroups a unit
// holds, LDS bytes, threads (dry runs: nothing is launched, no GPU is needed).
#include <cstdio>
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

int main()
{
    for (int dtype : {DT_F32, DT_BF16})
        for (int D : {64, 128}) {
            const std::string type = dtype == DT_F32 ? "f" : "t", dim = "Li" + std::to_string(D) + "E";
            TokenArgs a;
            std::memset(&a, 0, sizeof a);
            a.dtype = dtype; a.D = D; a.kv_heads = 2; a.b_hi = a.batch = 1; a.vocab = 1000;
            a.x = a.y = (void *)0x10000;         // aligned, never dereferenced
            a.cache.page_shift = 6;
            a.op = TK_CACHE_ATTENTION;
            for (int heads : {2, 8, 32})
                for (int S : {1, 3, 5, 8, 40, 300})
                    for (int pages : {1, 100, 2000}) {
                        a.heads = heads; a.S = S; a.cache.max_pages = pages;
                        const AttendGeom g = attend_geom(a);
                        tell(g.rows == 128 ? "cache_attention_wide_kernelI" + type + dim
                                           : "cache_attention_kernelI" + type + dim + "Li" + std::to_string(g.rows) + "ELi" + std::to_string(g.waves) + "E",
                             launch_cache_attention(a, nullptr, true, 1));
                        if (g.splits == 1) continue;
                        const LaunchInfo li = launch_cache_attention(a, nullptr, true, 2);
                        tell("cache_attention_join_kernelI" + type + dim + "Li" + std::to_string(li.lds_bytes ? 1024 / D : 1) + "E", li);
                    }
            a.heads = 8; a.S = 5; a.R = D;
            a.op = TK_CACHE_WRITE;
            tell("cache_write_kernelI" + type + dim, launch_cache_write(a, nullptr, true));
            a.op = TK_CACHE_READ;
            tell("cache_read_kernelI" + type + dim, launch_cache_read(a, nullptr, true));
            a.op = TK_SAMPLE;
            tell("sample_kernelI" + type + "E", launch_sample(a, nullptr, true, 0));
            a.op = TK_QKNORM_ROPE;
            for (int lanes = 1; lanes <= 64; lanes *= 2) {
                a.D = lanes * 8;
                tell("qknorm_rope_kernelI" + type + "Li" + std::to_string(lanes) + "E", launch_qknorm_rope(a, nullptr, true));
            }
        }
    return 0;
}
