// Sampling: one token per row of logits (gacer_sampling in include/gacer.h has the definition).
//
// A workgroup owns a row.  Weights are whole numbers, so every sum is exact and the same in any order, whatever adds it.  The entries that the
// filters keep are a prefix of the order "larger first, equal ones by index"; it ends at a key (the logit's bits in an order of
// unsigned numbers) and, among the entries with that key, at an index.
//   bf16 logits are few values: one pass over the row finds the largest and counts the entries by their 16 bits, in 65536 counters of 16 bits
// that fill 128 KB of LDS (entries that weigh nothing even against the largest so far are left out; they can only be kept where that changes
// no weight).  Scans over the counts, and over the counts times the weights of the some thousand values that occur, give the value at which top-k and
// the nucleus end and how many of its entries they still take.  The draw then adds the kept weights of the row, from a table, a part of
// the row per wave, and looks for its index in one of the parts; it reads again only pairs of vectors whose largest entry, noted by the first pass, is kept.
//   fp32 logits under top-k: the largest entries of the threads' shares give a value that at least k entries reach and few others do; those go
// into a list in LDS, and everything else happens on the list: ranks by counting, the nucleus by a scan over ranks, the draw by sums over smaller
// indexes.  Under top-p, or where k is large, a second pass puts every entry into one of 2048 bins by its distance from the largest, 1/64 of a
// temperature each (weights vanish 21.5 temperatures below), counting entries or adding weights; the bin in which the prefix ends is found by a
// scan, and few kept entries go into the list.  Otherwise only the last bin's entries need ranks, and the draw goes as for bf16.
//   Where a list would not hold its entries or a counter its count (a flat row), the prefix's end is found digit by digit of the key instead.
//
// What bounds it, and what it takes.  256 rows of 131072 bf16 logits under top-p and min-p (67 MB, 13 us at the rate of a large copy; one row in each unit):
// 51 us, which is the slowest row's time; an average row is done after 41.5: 7 until the counters are clear and the first loads there, 16 for the rest of the
// first pass, 8 for the scans of the counts, 1 for the table, 9 for the draw, one after another.  One row of 32000 fp32
// logits, top-k 50 and top-p: 11 us, a chain of two passes, some twenty barriers and instructions that a single workgroup runs through once; by bins
// 15, through the codes of bf16 as a first digit 21.
#include <hip/hip_runtime.h>
#include <algorithm>
#include "device_util.h"
#include "kernels.h"

namespace gacer {

typedef unsigned long long u64;

struct SampleArgs {
    const void *x;
    int64_t row_lo;
    int V;
    const float *u, *temperature, *top_p, *min_p;
    const int *top_k;
    int *tokens;
    float *logp;
};

static constexpr int MOST_ROWS = 1 << 21;               // of a launch: a grid holds fewer than 2^32 threads
static constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048, LIST = 2048, CODES = 32768, GROUPS = 512, PEAKS = 768;
// Entries that a list may hold where the alternative is another pass over the row: ranks by counting take n steps of a thread and more, a pass over 131072
// entries what 600 of them take.  By a list against without, one row: 388 entries of 128256 49 us against 62, 136 of 32000 19 against 22, 523 of 32000 24 either
// way (the line), 1243 of 32000 69 against 25; of a short row fewer would do, 397 of 8000 take 27 against 16.
static constexpr int SHORT = 512;

// numbers in an order of unsigned integers: -inf and NaN lowest, both zeros alike
__device__ __forceinline__ unsigned key_of(float x)
{
    if (x != x) x = -INFINITY;
    const unsigned b = __float_as_uint(x + 0.f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

__device__ __forceinline__ unsigned weight_of(float part) { return (unsigned)(part * 2147483648.f); }

// a logit that stands `d` temperatures (d <= 0) and a little below the top: no entry whose distance is d or more is smaller
__device__ __forceinline__ float below_top(float top, float temperature, float d) { return top + temperature * (d * 1.0001f - 0.001f); }
static constexpr float WEIGHTLESS = -22.f;             // 2^31 exp(d) < 1 from here down

// Weights of a row.  PLAIN: only a division is safe (a temperature very small or large, an infinite top).
template <bool PLAIN> struct Weights {
    float top, temperature, inverse, lowest;           // inverse: 1 / temperature, rounded; lowest: a distance at which every weight is 0
    __device__ Weights(float t, float temp) : top(t), temperature(temp), inverse(__fdiv_rn(1.f, temp)), lowest(-120.f * temp) {}
    // (x - top) / temperature, correctly rounded: a product with the rounded inverse is within two units in the last place, a step
    // with the exact remainder within one, and from there another step rounds correctly (no difference to a division in 4 x 2^30 pairs,
    // significands near one and two among them).  NaN counts as -inf.
    __device__ __forceinline__ float distance(float x) const
    {
        const float a = fmaxf(__fsub_rn(x, top), lowest);
        if constexpr (PLAIN) return x == top ? 0.f : __fdiv_rn(a, temperature);
        float q = __fmul_rn(a, inverse);
        q = __fmaf_rn(__fmaf_rn(-q, temperature, a), inverse, q);
        return __fmaf_rn(__fmaf_rn(-q, temperature, a), inverse, q);
    }
    __device__ __forceinline__ float part(unsigned key) const { return expf(distance(value_of(key))); }
    __device__ __forceinline__ float below(float d) const { return below_top(top, temperature, d); }
};
__device__ __forceinline__ int bin_of(float distance) { return min(BINS - 1, (int)(distance * -64.f)); }

// Sums over a wave, all lanes active, by moves within and between its rows of 16 lanes (a shuffle goes through LDS and takes ten times as long)
template <int MOVE, int ROWS> __device__ __forceinline__ u64 moved(u64 v)
{
    return (u64)(unsigned)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), MOVE, ROWS, 0xf, false) << 32 | (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, MOVE, ROWS, 0xf, false);
}
// sum over lanes 0..lane: lanes to the right by 1, 2, 4, 8 in a row, then a row's last lane to the next row, then lane 31 to the upper half
__device__ __forceinline__ u64 wave_scan(u64 v)
{
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane) { return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 wave_sum(u64 v) { return lane_of(wave_scan(v), 63); }
template <int MOVE, int ROWS> __device__ __forceinline__ float larger(float v)
{
    return fmaxf(v, __uint_as_float((unsigned)__builtin_amdgcn_update_dpp((int)0xFF800000u, (int)__float_as_uint(v), MOVE, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = larger<0x118, 0xf>(larger<0x114, 0xf>(larger<0x112, 0xf>(larger<0x111, 0xf>(v))));
    v = larger<0x143, 0xc>(larger<0x142, 0xa>(v));
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

struct Shared {
    u64 sums[WAVES], groups[GROUPS], before, all;
    unsigned equal[WAVES];
    float value;
    int entries, found;
    unsigned best, low;                                // keys of the largest logit so far, and of the lowest line from which entries were counted
    unsigned short peaks[WAVES][PEAKS];                // the upper 16 bits of the largest of each two vectors of a lane, in the order of the first pass
    union {
        unsigned codes[CODES];                         // entries by the code of their magnitude: positive ones in the upper half, negative ones in the lower
        struct {
            u64 bins[BINS], list[LIST];                // list: key, then the index's complement, so that larger numbers come first in the order
            unsigned weight[LIST];                     // of the list's entries, by rank
            int place[LIST];                           // and where they stand in it
        };
    };
};

template <typename T> struct Row {
    static constexpr int VEC = 16 / sizeof(T), DEPTH = 2, BATCH = 2;        // a lane's vectors in flight: of a pass (4: one row of 32000 fp32 11.5 us against 10.8, 8: 17.5), of the counting one
    const T *x;
    int V, head, vectors, per;                         // entries before the first 16-byte boundary, vectors after it, vectors of a wave's part

    __device__ void set(const T *row, int v)
    {
        x = row;
        V = v;
        head = min(v, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
        vectors = (v - head) / VEC;
        per = (vectors + WAVES - 1) / WAVES;
    }
    __device__ unsigned key(int i) const { return key_of(ld_f32(x, i)); }
    __device__ int part_begin(int w) const { return w == 0 ? 0 : head + min(w * per, vectors) * VEC; }
    __device__ int part_end(int w) const { return w == WAVES - 1 ? V : head + min((w + 1) * per, vectors) * VEC; }
    // f(index, logit) for the entries of the wave's part, DEPTH vectors of a lane in flight.  LONG: a body of many instructions stands there once per
    // element of a vector and not DEPTH times (what a wave runs through once comes from beyond the instruction cache).
    template <bool LONG = false, typename F> __device__ __forceinline__ void each(F f) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int b = min(vectors, (wave + 1) * per);
        const T *body = x + head;
        for (int v = wave * per + lane; v < b; v += 64 * DEPTH) {
            Vec<T, VEC> in[DEPTH];
#pragma unroll
            for (int k = 0; k < DEPTH; ++k) in[k] = ld_vec<T, VEC>(body, (int64_t)min(v + 64 * k, b - 1) * VEC);
            if constexpr (LONG) {
#pragma unroll 1
                for (int k = 0; k < DEPTH; ++k) {
                    if (v + 64 * k >= b) break;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f(head + (v + 64 * k) * VEC + e, in[0].get(e));
#pragma unroll
                    for (int j = 1; j < DEPTH; ++j) in[j - 1] = in[j];
                }
            } else {
#pragma unroll
                for (int k = 0; k < DEPTH; ++k) {
                    if (v + 64 * k >= b) break;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f(head + (v + 64 * k) * VEC + e, in[k].get(e));
                }
            }
        }
        if (border() >= 0) f(border(), ld_f32(x, border()));
    }
    // the lane's entry among those before and behind the vectors, -1: none
    __device__ __forceinline__ int border() const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, rest = V - head - vectors * VEC;
        return wave == 0 && lane < head ? lane : wave == WAVES - 1 && lane < rest ? V - rest + lane : -1;
    }
    // batches of BATCH vectors a lane in a wave's part
    __device__ int batches() const { return (per + 64 * BATCH - 1) / (64 * BATCH); }
    __device__ __forceinline__ void fetch(int turn, Vec<T, VEC> *in) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, b = min(vectors, (wave + 1) * per);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) in[k] = ld_vec<T, VEC>(x + head, (int64_t)max(0, min(wave * per + lane + (turn * BATCH + k) * 64, b - 1)) * VEC);
    }
    // The first pass over bf16 logits: the largest, its key in s.best; counters of the entries by value, but for those that weigh nothing even
    // against the largest so far; peaks of two vectors each.  `in`: the first batch.  Returns the number of the lane's counted entries.
    __device__ __forceinline__ unsigned count(Shared &s, float temperature, Vec<T, VEC> *in) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int first = wave * per + lane, b = min(vectors, (wave + 1) * per), turns = batches();
        unsigned counted = 0u;
        auto line = [&](float most) {                  // from which entries count
            most = wave_max(most);
            if (lane == 0) atomicMax(&s.best, key_of(most));
            const float from = fmaxf(below_top(value_of(*(volatile unsigned *)&s.best), temperature, WEIGHTLESS), -3.4028235e38f);
            if (lane == 0) atomicMin(&s.low, key_of(from));
            return from;
        };
        auto add = [&](float v, float from) {
            if (!(v >= from)) return;
            const unsigned bits = __float_as_uint(v + 0.f);              // both zeros alike
            atomicAdd((unsigned *)((char *)s.codes + ((bits >> 14) & 0x1FFFCu)), (int)bits < 0 ? 1u : 0x10000u);
            ++counted;
        };
        const bool peaked = turns * (BATCH * 32) <= PEAKS;
        auto batch = [&](int turn, const Vec<T, VEC> *in) {
            float peak[BATCH / 2], most = -INFINITY;
#pragma unroll
            for (int k = 0; k < BATCH / 2; ++k) {
                peak[k] = -INFINITY;
#pragma unroll
                for (int e = 0; e < VEC; ++e) peak[k] = fmaxf(peak[k], fmaxf(in[2 * k].get(e), in[2 * k + 1].get(e)));
                if (peaked) s.peaks[wave][(turn * (BATCH / 2) + k) * 64 + lane] = (unsigned short)(__float_as_uint(peak[k]) >> 16);
            }
#pragma unroll
            for (int k = 0; k < BATCH / 2; ++k) most = fmaxf(most, peak[k]);
            const float from = line(most);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                if (first + (turn * BATCH + k) * 64 >= b || !(peak[k / 2] >= from)) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) add(in[k].get(e), from);
            }
        };
        Vec<T, VEC> next[BATCH];
        for (int turn = 0; turn < turns; turn += 2) {  // one batch on its way while the other is counted
            fetch(turn + 1, next);
            batch(turn, in);
            if (turn + 1 == turns) break;
            fetch(turn + 2, in);
            batch(turn + 1, next);
        }
        if (__any(border() >= 0)) {
            const float mine = border() >= 0 ? ld_f32(x, border()) : -INFINITY;
            add(mine, line(mine));
        }
        return counted;
    }
    // f(logit) for the entries of the wave's part whose peak reaches `least`, and perhaps more
    template <typename F> __device__ __forceinline__ void each_above(const unsigned short *peaks, float least, F f) const
    {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = wave * per + lane, b = min(vectors, (wave + 1) * per);
        unsigned hits = 0u;
        for (int i = 0; i < batches() * (BATCH / 2); ++i)
            if (__uint_as_float((unsigned)peaks[i * 64 + lane] << 16) >= least) hits |= 1u << i;
        while (hits) {
            const int v = first + __builtin_ctz(hits) * 128;
            hits &= hits - 1;
            Vec<T, VEC> in[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) in[k] = ld_vec<T, VEC>(x + head, (int64_t)min(v + 64 * k, b - 1) * VEC);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (v + 64 * k >= b) break;
#pragma unroll
                for (int e = 0; e < VEC; ++e) f(in[k].get(e));
            }
        }
        if (border() >= 0) f(ld_f32(x, border()));
    }
};

__device__ __forceinline__ u64 entry_of(unsigned key, int i) { return (u64)key << 32 | (unsigned)~i; }
__device__ __forceinline__ unsigned entry_key(u64 e) { return (unsigned)(e >> 32); }
__device__ __forceinline__ int entry_index(u64 e) { return (int)~(unsigned)e; }

__device__ __forceinline__ u64 goal_of(float u, u64 total)
{
    const double goal = floor((double)u * (double)total);
    return goal > 0. ? (goal >= (double)total ? total - 1 : (u64)goal) : 0;
}

// sum over the workgroup
__device__ u64 block_sum(Shared &s, u64 v)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.sums[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 all = 0;
    for (int w = 0; w < WAVES; ++w) all += s.sums[w];
    return all;
}

// The first bin, from 0 on, at which the sum passes the line: done(sum up to and with it).  `before` receives the sum in front of it.
template <typename D> __device__ int first_bin(Shared &s, D done, u64 *before)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const u64 a = s.bins[2 * tid], b = s.bins[2 * tid + 1];
    u64 v = wave_scan(a + b);
    __syncthreads();
    if (lane == 63) s.sums[wave] = v;
    if (tid == 0) s.found = BINS - 1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += s.sums[w];
    if (done(v) && !done(v - a - b)) {
        const bool first = done(v - b);
        s.found = 2 * tid + (first ? 0 : 1);
        s.before = first ? v - a - b : v - b;
    }
    __syncthreads();
    *before = s.before;
    return s.found;
}

// bf16 values in the order of unsigned 16-bit numbers
__device__ __forceinline__ unsigned key16_of(float x)
{
    const unsigned h = __float_as_uint(x + 0.f) >> 16;
    return h ^ (h & 0x8000u ? 0xFFFFu : 0x8000u);
}
__device__ __forceinline__ float value16_of(unsigned k) { return __uint_as_float((k & 0x8000u ? k ^ 0x8000u : k ^ 0xFFFFu) << 16); }

// group of the value with these upper bits of magnitude, see first_value()
__device__ __forceinline__ int group_of(float x)
{
    const unsigned b = __float_as_uint(x);
    const int m = (int)(b >> 23 & 255u);
    return b >> 31 ? GROUPS / 2 + m : GROUPS / 2 - 1 - m;
}

// The largest value up to and with which the measure of the counted entries, from the largest value on, reaches the line; `before` receives the measure
// of larger ones, `all` of the row, `counted` the sum of the counts.  measure(value, entries) of a value; reached(measure, all).  Groups of 128 values (a
// power of two and a sign) are added by a wave each, then scanned; the first 256 groups are those of the positive values.  `range`: first and last
// group that holds any.
template <typename M, typename D> __device__ __forceinline__ float first_value(Shared &s, int2 range, M measure, D reached, u64 *before, u64 *all, u64 *counted)
{
    constexpr int HALF = GROUPS / 2;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    // the lane's two counters of a group, of the larger value first: magnitudes of positive values fall, of negative ones rise
    auto counters = [&](int group) {
        const int m = group < HALF ? (HALF - 1 - group) * 128 + 126 - 2 * lane : (group - HALF) * 128 + 2 * lane;
        const uint2 c = *(const uint2 *)&s.codes[m];
        return group < HALF ? make_uint2(c.y >> 16, c.x >> 16) : make_uint2(c.x & 0xFFFFu, c.y & 0xFFFFu);
    };
    auto value = [&](int group, int which) {
        const int m = group < HALF ? (HALF - 1 - group) * 128 + 127 - 2 * lane - which : (group - HALF) * 128 + 2 * lane + which;
        return __uint_as_float((unsigned)m << 16 | (group < HALF ? 0u : 0x80000000u));
    };
    __syncthreads();                                   // all have read what stands in s.sums and s.groups
    for (int i = tid; i < GROUPS; i += THREADS) s.groups[i] = 0;
    __syncthreads();
    unsigned entries = 0u;
    for (int g = range.x + ((wave - range.x) & (WAVES - 1)); g <= range.y; g += WAVES) {
        const uint2 n = counters(g);
        if (!__any((n.x | n.y) != 0u)) continue;
        entries += n.x + n.y;
        u64 v = 0;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const unsigned c = k ? n.y : n.x;
            if (c) v += measure(value(g, k), c);
        }
        v = wave_sum(v);
        if (lane == 0) s.groups[g] = v;
    }
    const u64 in_wave = wave_sum(entries);
    if (lane == 0) s.sums[wave] = in_wave;
    __syncthreads();
    if (wave == 0) {
        u64 part[GROUPS / 64], v = 0;                  // eight groups of a lane
#pragma unroll
        for (int i = 0; i < GROUPS / 64; ++i) {
            part[i] = s.groups[lane * (GROUPS / 64) + i];
            v += part[i];
        }
        const u64 upto = wave_scan(v), total = lane_of(upto, 63);
        u64 sum = upto - v, at = 0;
        int g = 0;
        bool found = false;
#pragma unroll
        for (int i = 0; i < GROUPS / 64; ++i) {
            if (!found && reached(sum + part[i], total)) {
                found = true;
                g = i;
                at = sum;
            }
            sum += part[i];
        }
        const u64 mine = __ballot(found);
        const int l = mine ? __builtin_ctzll(mine) : 63;
        g = l * (GROUPS / 64) + __builtin_amdgcn_readlane(g, l);
        at = lane_of(at, l);
        const uint2 n = counters(g);
        const u64 x = n.x ? measure(value(g, 0), n.x) : 0, y = n.y ? measure(value(g, 1), n.y) : 0, in = at + wave_scan(x + y);
        const u64 hit = __ballot(reached(in, total));
        if (lane == (hit ? __builtin_ctzll(hit) : 63)) {
            const bool first = reached(in - y, total);
            s.value = value(g, first ? 0 : 1);
            s.before = first ? in - y - x : in - y;
            s.all = total;
        }
    }
    __syncthreads();
    *before = s.before;
    *all = s.all;
    *counted = 0;
    for (int w = 0; w < WAVES; ++w) *counted += s.sums[w];
    return s.value;
}

// entries of the list in order: place[r] and weight[r] of rank r
template <typename W> __device__ void rank_list(Shared &s, const W &w, int n)
{
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const u64 me = s.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += s.list[j] > me;
        s.place[rank] = i;
        s.weight[rank] = weight_of(w.part(entry_key(me)));
    }
    __syncthreads();
}

// The number of ranks, at most n, up to and with the first at which `before` and the weights so far reach the line; by one wave, told to all.
__device__ int ranks_to(Shared &s, int n, u64 before, double reach)
{
    if (threadIdx.x < 64) {
        int r = n;
        for (int i = 0; i < n; i += 64) {
            const int at = i + (int)threadIdx.x;
            const u64 v = before + wave_scan(at < n ? s.weight[at] : 0u);
            const u64 hit = __ballot(at < n && (double)v >= reach);
            if (hit) {
                r = i + __builtin_ctzll(hit) + 1;
                break;
            }
            before = lane_of(v, 63);
        }
        if (threadIdx.x == 0) s.found = r;
    }
    __syncthreads();
    return s.found;
}

// end of the kept prefix by the digits of the key, for rows whose entries crowd in one bin
template <typename T, typename M> __device__ void prefix_by_digits(Shared &s, const Row<T> &row, double reach, M measure, unsigned &cut, int &last)
{
    const int tid = threadIdx.x;
    u64 before = 0;                                    // measure of the keys above the digits found so far
    unsigned prefix = 0u;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) s.bins[tid] = 0;
        __syncthreads();
        row.each([&](int i, float x) {
            const unsigned k = key_of(x);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
                const u64 m = measure(i, k);
                if (m) atomicAdd(&s.bins[(k >> shift) & 255u], m);
            }
        });
        __syncthreads();
        int digit = 255;
        for (; digit > 0 && (double)(before + s.bins[digit]) < reach; --digit) before += s.bins[digit];
        prefix |= (unsigned)digit << shift;
    }
    // entries of this very key are taken by index until the line is reached: halve in on the last one's index
    auto same = [&](int i, unsigned k) -> u64 { return k == prefix ? measure(i, k) : 0; };
    int lo = 0, hi = row.V;                            // the last one lies in [lo, hi)
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        u64 v = 0;
        for (int i = lo + tid; i < mid; i += THREADS) v += same(i, row.key(i));
        v = block_sum(s, v);
        if ((double)(before + v) >= reach) hi = mid;
        else {
            before += v;
            lo = mid;
        }
    }
    cut = prefix;
    last = lo;
}

struct Filters { float top_p, min_p, u; int top_k; };

// The draw from a list that holds every kept entry (and perhaps more): the first n ranks, of them those of at least min_p
template <typename W, typename F> __device__ void draw_from_list(Shared &s, const W &w, const Filters &f, int n, F write)
{
    const int tid = threadIdx.x;
    u64 v = 0;
    for (int i = tid; i < n; i += THREADS) {
        const u64 e = s.list[s.place[i]];
        const unsigned m = i == 0 || w.part(entry_key(e)) >= f.min_p ? s.weight[i] : 0u;
        s.bins[i] = (u64)(unsigned)entry_index(e) << 32 | m;
        v += m;
    }
    const u64 total = block_sum(s, v), goal = goal_of(f.u, total);
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {           // whose weight does the goal fall on, smaller indexes before it
        const u64 me = s.bins[i];
        u64 sum = 0;
        for (int j = 0; j < n; ++j) sum += (s.bins[j] >> 32) < (me >> 32) ? (unsigned)s.bins[j] : 0u;
        if (sum <= goal && goal < sum + (unsigned)me) write((int)(me >> 32), value_of(entry_key(s.list[s.place[i]])), total);
    }
}

// What the draw needs to know of a kept set: weights, by value, of entries above `cut`, and `ties` entries, by index, that equal it.  Sums over
// the waves' parts of the row, then over threads within the part that the goal falls into, then one by one.
template <bool LONG, typename T, typename K, typename F> __device__ __forceinline__ void draw_from_row(Shared &s, const Row<T> &row, bool peaked, float u, float least, float cut, u64 ties, unsigned of_cut, K weight, F write)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    // entries below `least` (which is not below `cut`) weigh nothing
    auto add = [&](float x, u64 &sum, unsigned &equal) {
        if (!(x >= least)) return;
        if (x > cut) sum += weight(x);
        else ++equal;
    };
    u64 v = 0;
    unsigned n = 0;
    if (peaked) row.each_above(s.peaks[wave], least, [&](float x) { add(x, v, n); });
    else row.template each<LONG>([&](int, float x) { add(x, v, n); });
    v = wave_sum(v);
    n = (unsigned)wave_sum(n);
    __syncthreads();
    if (lane == 0) {
        s.sums[wave] = v;
        s.equal[wave] = n;
    }
    __syncthreads();
    u64 total = 0, all = 0;
    for (int k = 0; k < WAVES; ++k) {
        total += s.sums[k];
        all += s.equal[k];
    }
    ties = all < ties ? all : ties;
    total += ties * of_cut;
    u64 goal = goal_of(u, total);
    int p = 0;
    for (; p < WAVES - 1; ++p) {
        const u64 taken = s.equal[p] < ties ? s.equal[p] : ties, part = s.sums[p] + taken * of_cut;
        if (goal < part) break;
        goal -= part;
        ties -= taken;
    }
    const int lo = row.part_begin(p), hi = row.part_end(p), each = (hi - lo + THREADS - 1) / THREADS;
    const int b = min(hi, lo + tid * each), e = min(hi, b + each);
    v = 0;
    n = 0;
    constexpr int TOGETHER = 8;
    auto load = [&](int i, float *in) {
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) in[k] = ld_f32(row.x, min(i + k, row.V - 1));
    };
    for (int i = b; i < e; i += TOGETHER) {
        float in[TOGETHER];
        load(i, in);
        if constexpr (LONG) {
#pragma unroll 1
            for (int k = 0; k < TOGETHER; ++k) {
                if (i + k < e) add(in[0], v, n);
#pragma unroll
                for (int j = 1; j < TOGETHER; ++j) in[j - 1] = in[j];
            }
        } else {
#pragma unroll
            for (int k = 0; k < TOGETHER; ++k)
                if (i + k < e) add(in[k], v, n);
        }
    }
    u64 sum = wave_scan(v), equal = wave_scan(n);
    __syncthreads();
    if (lane == 63) {
        s.sums[wave] = sum;
        s.equal[wave] = (unsigned)equal;
    }
    __syncthreads();
    for (int k = 0; k < wave; ++k) {
        sum += s.sums[k];
        equal += s.equal[k];
    }
    auto upto = [&](u64 sums, u64 equals) { return sums + (equals < ties ? equals : ties) * of_cut; };
    if (upto(sum, equal) > goal && upto(sum - v, equal - n) <= goal) {
        sum -= v;
        equal -= n;
        float in[TOGETHER] = {};
        for (int i = b; i < e; ++i) {
            if (((i - b) & (TOGETHER - 1)) == 0) load(i, in);
            unsigned one = 0;
            add(in[0], sum, one);
            equal += one;
            if (upto(sum, equal) > goal) {
                write(i, in[0], total);
                break;
            }
#pragma unroll
            for (int j = 1; j < TOGETHER; ++j) in[j - 1] = in[j];
        }
    }
}

// mine: the largest logit that the thread has seen (fp32); `coded`: the entries have been counted by their values (bf16); `counted`: how many of them there are
template <typename T, bool PLAIN> __device__ __forceinline__ void sample_row(const SampleArgs &a, Shared &s, const Row<T> &row, int64_t r, float top, float temperature, Filters f, float mine, bool coded, u64 counted)
{
    const int tid = threadIdx.x;
    const Weights<PLAIN> w(top, temperature);
    const unsigned none = key_of(-INFINITY);
    auto write = [&](int token, float x, u64 total) {
        a.tokens[r] = token;
        if (a.logp) a.logp[r] = w.distance(x) - logf((float)total * 0x1p-31f);
    };
    auto full = [&](float x) { return weight_of(expf(w.distance(x))); };           // before min_p
    auto kept = [&](float x) {
        const float part = expf(w.distance(x));
        return part >= f.min_p || x == top ? weight_of(part) : 0u;
    };
    // a logit below which nothing is kept, whatever the other filters say: min_p, and weights of 0 (21.5 temperatures below)
    const float floor_p = w.below(f.min_p > 0.f ? logf(f.min_p) : WEIGHTLESS);

    if constexpr (sizeof(T) == 2) {
        // 16 bits hold a counter unless more than 65535 entries are alike; then the counts add up to less than there are
        u64 before, all;
        float cut = -INFINITY;
        u64 ties = 0;
        const u64 finite = counted;
        const int2 range = make_int2(group_of(top), group_of(value_of(s.low)));
        if (coded && f.top_k < a.V) {
            const u64 k64 = (u64)f.top_k;
            const float v = first_value(s, range, [](float, unsigned n) -> u64 { return n; }, [&](u64 m, u64) { return m >= k64; }, &before, &all, &counted);
            if (all >= k64) {                          // otherwise top-k keeps every finite entry
                cut = v;
                ties = k64 - before;
            }
        }
        const float cut_k = cut;
        const u64 ties_k = ties;
        if (coded && counted == finite && f.top_p < 1.f) {
            const double p = (double)f.top_p;
            auto entries = [&](float x, unsigned n) -> unsigned { return x > cut_k ? n : x == cut_k ? (unsigned)ties_k : 0u; };
            cut = first_value(s, range, [&](float x, unsigned n) -> u64 { return (u64)full(x) * entries(x, n); }, [&](u64 m, u64 t) { return m != 0 && (double)m >= p * (double)t; }, &before, &all, &counted);
            const double reach = p * (double)all;
            const u64 each = full(cut);
            ties = 1;
            if (each) {                                // the fewest with which the line is reached
                ties = (u64)((reach - (double)before) / (double)each);
                while ((double)(before + ties * each) < reach) ++ties;
                while (ties > 1 && (double)(before + (ties - 1) * each) >= reach) --ties;
            }
        }
        coded = coded && counted == finite;
        if (coded) {
            const float least = fmaxf(fmaxf(cut, value_of(none + 1u)), floor_p);
            const unsigned high = key16_of(top), span = high - key16_of(least);
            const unsigned of_cut = kept(cut);
            ties = least > cut ? 0 : ties;
            if (span < (unsigned)CODES) {              // a table of the kept values' weights, where the counts were
                __syncthreads();
#pragma unroll 1
                for (unsigned i = tid; i <= span; i += THREADS) s.codes[i] = kept(value16_of(high - i));
                __syncthreads();
                draw_from_row<false>(s, row, row.batches() * (Row<T>::BATCH * 32) <= PEAKS, f.u, least, cut, ties, of_cut, [&](float x) { return s.codes[high - key16_of(x)]; }, write);
            } else draw_from_row<true>(s, row, false, f.u, least, cut, ties, of_cut, kept, write);
            return;
        }
    }
    auto clear = [&] {
        __syncthreads();
        for (int i = tid; i < BINS; i += THREADS) s.bins[i] = 0;
        __syncthreads();
    };
    // entries of at least `least`, and `in(x, i)`, into the list; their number, which may be more than it holds
    auto gather = [&](float least, auto in) {
        __syncthreads();
        if (tid == 0) s.entries = 0;
        __syncthreads();
        row.each([&](int i, float x) {
            if (x < least || !in(x, i)) return;
            const int at = atomicAdd(&s.entries, 1);
            if (at < LIST) s.list[at] = entry_of(key_of(x), i);
        });
        __syncthreads();
        return s.entries;
    };
    auto bin_floor = [&](int bin) { return bin < BINS - 1 ? w.below((bin + 1) * (-1.f / 64.f)) : -INFINITY; };

    unsigned cut = 0u;                                 // kept: keys above `cut`, and those equal to it up to index `last`
    int last = a.V;
    if (f.top_k < a.V) {
        u64 before;
        const u64 k64 = (u64)f.top_k;
        auto to_bin = [&](float x) {
            const int bin = bin_of(w.distance(x));
            if (bin < BINS - 1) atomicAdd(&s.bins[bin], 1ull);
        };
        auto draw = [&](int n) {
            rank_list(s, w, n);
            int first = f.top_k;
            if (f.top_p < 1.f) {
                u64 v = 0;
                for (int i = tid; i < first; i += THREADS) v += s.weight[i];
                first = ranks_to(s, first, 0, (double)f.top_p * (double)block_sum(s, v));
            }
            draw_from_list(s, w, f, first, write);
        };
        if (sizeof(T) == 4 && f.top_k <= THREADS / 4) {
            // the k largest entries are no smaller than the k largest of the threads' largest ones, and few others are.  Against the bins, us: one row of 32000
            // 11.0 and 14.7 with k = 50, 19.4 and 22.7 with 256, 26 and 28 with 384, but 34 and 32 with 500, 118 and 65 with 900; of 5000 9.0 and 9.9, 15.7 and 16.4,
            // 20.6 and 20.8, 29 and 25, 150 and 54; of 128256 18 and 32, 27 and 41, 33 and 46, 44 and 51, 104 and 87; 64 rows of each alike
            clear();
            to_bin(mine);
            __syncthreads();
            const int bin = first_bin(s, [&](u64 v) { return v >= k64; }, &before);
            if (bin < BINS - 1) {
                const float least = bin_floor(bin);
                const int n = gather(least, [](float, int) { return true; });
                if (n <= LIST) {
                    draw(n);
                    return;
                }
            }
        }
        clear();
        // the last bin takes the far end of the row; it is not counted one by one, at one address, but taken to hold everything
        row.each([&](int, float x) { to_bin(x); });
        if (tid == 0) s.bins[BINS - 1] = (u64)a.V;
        __syncthreads();
        const int bin = first_bin(s, [&](u64 v) { return v >= k64; }, &before);
        if (before + s.bins[bin] <= LIST) {
            draw(gather(bin_floor(bin), [&](float x, int) { return bin_of(w.distance(x)) <= bin; }));
            return;
        }
        prefix_by_digits(s, row, (double)f.top_k, [&](int, unsigned) -> u64 { return 1; }, cut, last);
    }
    if (f.top_p < 1.f) {
        const unsigned cut_k = cut;
        const int last_k = last;
        auto allowed = [&](int i, unsigned k) { return k > cut_k || (k == cut_k && i <= last_k); };
        auto measure = [&](int i, unsigned k) -> u64 { return allowed(i, k) ? weight_of(w.part(k)) : 0u; };
        clear();
        if (cut_k == 0u)
            row.each([&](int, float x) {
                const float q = w.distance(x);
                const unsigned m = weight_of(expf(q));
                if (m) atomicAdd(&s.bins[bin_of(q)], (u64)m);
            });
        else
            row.each([&](int i, float x) {
                const u64 m = measure(i, key_of(x));
                if (m) atomicAdd(&s.bins[bin_of(w.distance(x))], m);
            });
        __syncthreads();
        u64 all = 0, before;
        for (int i = tid; i < BINS; i += THREADS) all += s.bins[i];
        const double reach = (double)f.top_p * (double)block_sum(s, all);
        const int bin = first_bin(s, [&](u64 v) { return (double)v >= reach; }, &before);
        // few kept entries (min_p, or a peaked row): all of them go into the list.  How many they are follows from the bins, whose entries weigh
        // the same within 1/64.
        const float least = fmaxf(bin_floor(bin), floor_p);
        const int last_bin = min(bin, bin_of(w.distance(least)));
        float many = 0.f;
        for (int i = tid; i <= last_bin; i += THREADS) many += (float)s.bins[i] * 0x1p-31f * expf((i + 0.5f) * (1.f / 64.f));
        if (block_sum(s, (u64)(many * 1024.f)) >> 10 < (u64)(SHORT - SHORT / 16)) {
            const int n = gather(least, [&](float x, int i) { return allowed(i, key_of(x)); });
            if (n <= LIST) {
                rank_list(s, w, n);
                draw_from_list(s, w, f, ranks_to(s, n, 0, reach), write);
                return;
            }
        }
        const int m = gather(bin_floor(bin), [&](float x, int i) { return bin_of(w.distance(x)) == bin && allowed(i, key_of(x)); });
        if (m <= LIST) {
            rank_list(s, w, m);
            const u64 e = s.list[s.place[max(1, ranks_to(s, m, before, reach)) - 1]];
            cut = entry_key(e);
            last = entry_index(e);
        } else prefix_by_digits(s, row, reach, measure, cut, last);
    }
    // entries that equal the last one, up to it
    const float value = cut > none ? value_of(cut) : -INFINITY;
    u64 ties = 0;
    if (cut > none) {
        for (int i = tid; i <= min(last, a.V - 1); i += THREADS) ties += row.key(i) == cut;
        ties = block_sum(s, ties);
    }
    const float least = fmaxf(fmaxf(value, value_of(none + 1u)), floor_p);
    draw_from_row<true>(s, row, false, f.u, least, value, least > value ? 0 : ties, kept(value), kept, write);
}

template <typename T> __global__ __launch_bounds__(1024) void sample_kernel(SampleArgs a)
{
    __shared__ Shared s;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t r = a.row_lo + blockIdx.x;
    Row<T> row;
    row.set((const T *)a.x + r * a.V, a.V);
    // on their way while the row's filters are fetched and the counters cleared
    Vec<T, Row<T>::VEC> in[sizeof(T) == 2 ? Row<T>::BATCH : 1];
    if constexpr (sizeof(T) == 2) {
        if (row.vectors) row.fetch(0, in);
    }
    const float temperature = a.temperature ? a.temperature[r] : 1.f;
    Filters f = {a.top_p ? a.top_p[r] : 1.f, a.min_p ? a.min_p[r] : 0.f, a.u[r], a.top_k ? a.top_k[r] : 0};
    if (f.top_k <= 0 || f.top_k > a.V) f.top_k = a.V;
    const bool one = f.top_k == 1 || !(temperature > 0.f) || !(f.top_p > 0.f) || !(f.min_p <= 1.f);       // the first of the largest
    const bool coded = sizeof(T) == 2 && !one && (f.top_k < a.V || f.top_p < 1.f);
    float top = -INFINITY;
    unsigned counted = 0u;
    if constexpr (sizeof(T) == 2) {
        if (coded) {
            for (int i = tid * 4; i < CODES; i += THREADS * 4) *(uint4 *)&s.codes[i] = make_uint4(0u, 0u, 0u, 0u);
            if (tid == 0) {
                s.best = key_of(-INFINITY);
                s.low = ~0u;
            }
            __syncthreads();
            counted = row.count(s, temperature, in);
        }
    }
    if (sizeof(T) == 4 || !coded) row.each([&](int, float x) { top = fmaxf(top, x); });
    const float mine = top;
    top = wave_max(top);
    const u64 in_wave = wave_sum(counted);
    if (lane == 0) s.sums[wave] = (in_wave << 32) | __float_as_uint(top);
    __syncthreads();
    u64 finite = 0;
    for (int w = 0; w < WAVES; ++w) {
        top = fmaxf(top, __uint_as_float((unsigned)s.sums[w]));
        finite += s.sums[w] >> 32;
    }
    if (coded) top = value_of(s.best);
    top += 0.f;
    if (top == -INFINITY) {
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logp) a.logp[r] = -INFINITY;
        }
        return;
    }
    if (one) {
        int first = a.V;
        row.each([&](int i, float x) { if (x == top) first = min(first, i); });
        for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
        __syncthreads();
        if (lane == 0) s.sums[wave] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < WAVES; ++w) first = min(first, (int)s.sums[w]);
            a.tokens[r] = first;
            if (a.logp) a.logp[r] = 0.f;
        }
        return;
    }
    if (temperature > 1e-18f && temperature < 1e18f && top < INFINITY) sample_row<T, false>(a, s, row, r, top, temperature, f, mine, coded, finite);
    else sample_row<T, true>(a, s, row, r, top, temperature, f, mine, coded, finite);
}

LaunchInfo launch_sample(const TokenArgs &a, hipStream_t s, bool dry, int)
{
    SampleArgs b;
    b.x = a.x; b.row_lo = (int64_t)a.b_lo * a.S; b.V = a.vocab; b.u = a.u; b.temperature = a.temperature; b.top_p = a.top_p; b.min_p = a.min_p;
    b.top_k = a.top_k; b.tokens = a.tokens; b.logp = a.logp;
    LaunchInfo li;
    li.workgroups = (a.b_hi - a.b_lo) * a.S;
    li.threads = THREADS; li.lds_bytes = (int)sizeof(Shared); li.wg_per_cu = 1; li.kernel = a.dtype == DT_BF16 ? "sample_bf16" : "sample_f32"; li.phases = 1;
    if (dry || !li.workgroups) return li;
    for (int at = 0; at < li.workgroups; at += MOST_ROWS, b.row_lo += MOST_ROWS) {
        const dim3 grid(std::min(li.workgroups - at, MOST_ROWS));
        if (a.dtype == DT_BF16) GACER_LAUNCH(sample_kernel<unsigned short>, grid, dim3(THREADS), 0, s, b);
        else GACER_LAUNCH(sample_kernel<float>, grid, dim3(THREADS), 0, s, b);
    }
    return li;
}

}  // namespace gacer
