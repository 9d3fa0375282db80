// One token per row of logits, drawn with the caller's random numbers (onela_sample_tokens).
//
// With w_i = exp((x_i - max) / T) and the tokens ordered by (x descending, index ascending), top-k, top-p and min-p each keep a
// leading run of that order, so all of them together keep a leading run too, and no sort is needed: what is kept is everything above one
// value, and the first m (by index) of the tokens that have that value.  The token is where the running sum of the kept masses, in the order of
// indices, passes uniform * sum.
//
// A row lies in the shared memory of one cluster of 1 to 8 CTAs, read from memory once.  Masses are integers, w in units of 2^-F with F = 62 -
// ceil(log2 vocab) (43 places or more), so sums are exact in any order, atomics included.  w = 2^(n / 256 + f / 256) in 64 bits, |f| <= 1 / 2:
// 2^(n mod 256 / 256) from a table, the rest by its series to the third power (Tang 1989; relative error 2e-13).  (64 rows of 100 003 logits without
// filters take 9 us more than a pass that only looks for the largest; the same on sums of two fp32 numbers, 36 instructions, 21, with the conversions
// from and to 64 bits done on the bits 14.)
//   top-k   tokens counted by bins of their distance from the largest (896 of them); the bin in which the count passes k is cut
//           into 512 bins of the values' bit patterns, and so on until a bin holds one token or one value
//   top-p   the same descent on the bins' masses, from the same first histogram, towards top_p times the mass of the top-k tokens.  (Counts alone in the
//           first histogram, the masses around a guessed bin by a pass of their own: 86 us against 69 for 64 rows of 100 003.)
// A histogram is reduced by the cluster (a CTA sums a share of the bins over all CTAs and hands the sums to all), two cluster barriers.
// The draw: kept masses by warps (a warp has a run of neighbours), then the one run that passes the target token by token.
// What bounds it: launches of a few rows the chain of barriers (one row of 131 072 with top-k and top-p 29 us, 11.5 without filters; the code, which a launch runs
// once, counts: loops rolled, 152 -> 128 KB, took 2 us off), many rows the
// exponentials' and the histogram's instructions (64 rows of 100 003: 13 us to find the largest, 22 without filters, 64 with top-p and min-p).
#include <cooperative_groups.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <mutex>

#include "onela_internal.h"
#include "onela_layout.cuh"

namespace onela {
namespace {

namespace cg = cooperative_groups;
using u64 = unsigned long long;

constexpr int MAX_THREADS = 1024, TABLE = 256, BINS = 896, FINE = 512, MAX_SLICE = 50048, MAX_CLUSTER = 8, MAX_VOCAB = 360000;
constexpr float BINS_PER_UNIT = 32.f;            // first histogram: bins of 1 / 32 up to 28 below the largest, the rest in the last one

struct SampleArgs {
    const void* logits;
    const float *uniforms, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* tokens;
    float* logprobs;
    long long stride;
    int32_t vocab, places;                       // places: F
    int32_t histograms;                          // shared memory has room for them
};

// The first histogram has BINS bins, finer ones FINE.  (As small as this so that two CTAs hold 100 000 fp32 logits: by four 64 rows are
// two waves, 101 us instead of 74.)
struct Histograms {
    uint32_t count[BINS], low[BINS], high[BINS];      // this CTA's; a mass's two halves
    u64 all_mass[BINS], fine_mass[FINE];              // the cluster's, of the first and of a finer one
    uint32_t all_count[BINS], fine_count[FINE];
};

// What every CTA of a row knows.
struct Row {
    float largest, zero_from;                    // what lies below zero_from has no mass
    double scale;                                // 256 log2(e) / T
    int places;                                  // F
    bool greedy;
};

// bit pattern in the order of the values (-0 has been made +0, NaN -inf)
template <typename T>
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x), k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return sizeof(T) == 2 ? k >> 16 : k;         // (bf16: the lower half says nothing)
}
__device__ __forceinline__ int first_bin(const Row& r, float x) { return min(BINS - 1, (int)((r.largest - x) * BINS_PER_UNIT)); }
// The weight in units of 2^-F: 2^F at the largest, 0 at -inf.  table[j] = 2^(j / 256).
__device__ __forceinline__ u64 mass(const Row& r, const double* table, float x) {
    constexpr double MAGIC = 0x1.8p52, LN2 = 0x1.62e42fefa39efp-9;                      // (ln 2 / 256)
    // (the difference first: scale times either side of it would leave the difference their rounding, 1e-9 of a mass where logits are 10^7 temperatures from 0)
    const double d = (double)x - (double)r.largest, t = fma(d, r.scale, MAGIC), f = fma(d, r.scale, MAGIC - t) * LN2;
    const int n = __double2loint(t);
    const double w = table[n & (TABLE - 1)], v = fma(w, f * fma(f, fma(f, 1.0 / 6.0, 0.5), 1.0), w);
    const u64 m = __double2ull_rn(__hiloint2double(__double2hiint(v) + ((n >> 8) + r.places) * (1 << 20), __double2loint(v)));
    return x == r.largest ? 1ull << r.places : x < r.zero_from ? 0 : m;
}

// The end of the kept run: tokens of first bin `bin` whose keys lie in [low, high] are its last ones, `ties` of them (by index) kept; what
// lies above is kept whole.  No token of the bin lies outside [from, to].
struct Cut {
    int bin;                                     // -1: everything is above
    float from, to;
    uint32_t low, high, ties;
};
// values that a bin can hold, half a bin more on either side (the bin of a value is off by far less)
__device__ __forceinline__ float bin_from(const Row& r, int b) {
    return b >= BINS - 1 || isinf(r.largest) ? -INFINITY : (float)((double)r.largest - (b + 1.5) / BINS_PER_UNIT);
}
__device__ __forceinline__ float bin_to(const Row& r, int b) { return isinf(r.largest) ? INFINITY : (float)((double)r.largest - (b - 0.5) / BINS_PER_UNIT); }
// 1 above, 0 at the end of the run, -1 below
template <typename T>
__device__ __forceinline__ int side(const Row& r, const Cut& c, float x) {
    const int b = first_bin(r, x);
    const uint32_t k = key_of<T>(x);
    const int within = k > c.high ? 1 : k >= c.low ? 0 : -1;
    return c.bin < 0 || b < c.bin ? 1 : b > c.bin ? -1 : within;
}

template <typename X>
__device__ __forceinline__ X block_exclusive_scan(X x, X* warp_s, X* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    X run = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const X y = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += y;
    }
    __syncthreads();                             // warp_s is free
    if (lane == 31) warp_s[warp] = run;
    __syncthreads();
    const X own = lane < warps ? warp_s[lane] : 0;
    X sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const X y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
    }
    *total = __shfl_sync(0xffffffffu, sum, 31);
    return __shfl_sync(0xffffffffu, sum - own, warp) + run - x;
}

template <typename T>
__global__ void __launch_bounds__(MAX_THREADS) sample_kernel(const SampleArgs a) {
    constexpr int VE = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ double table_s[TABLE];
    __shared__ u64 scan64_s[MAX_THREADS / 32];
    __shared__ uint32_t scan32_s[MAX_THREADS / 32];
    __shared__ float largest_s, warp_largest_s[MAX_THREADS / 32];
    __shared__ u64 total_mass_s, tie_mass_s;
    __shared__ uint32_t total_ties_s, run_ties_s[32];
    __shared__ u64 run_sum_s[32], run_tie_mass_s[32];
    __shared__ int run_found_s;
    __shared__ int found_bin_s;
    __shared__ u64 found_mass_s, found_before_s;
    __shared__ u64 part_s[MAX_THREADS / 32][4], cta_part_s[2][4], row_part_s[4];
    __shared__ uint32_t found_count_s;
    const cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks(), tid = threadIdx.x, threads = blockDim.x;
    const long long row = blockIdx.x / ctas;
    auto sync = [&] {
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    };
    Histograms* hist = reinterpret_cast<Histograms*>(smem);
    float* x_s = reinterpret_cast<float*>(smem + (a.histograms ? sizeof(Histograms) : 0));
    for (int j = tid; j < TABLE; j += threads) table_s[j] = exp2(j * (1.0 / TABLE));
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- the slice: elements counted from the 16-byte boundary at or before the row's first ----
    const T* p = static_cast<const T*>(a.logits) + row * a.stride;
    const int skip = (int)(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
    const long long end = (long long)skip + a.vocab;
    const int units = (int)((end + VE - 1) / VE), each = (units + ctas - 1) / ctas;
    const int unit0 = min(units, rank * each), n = (min(units, unit0 + each) - unit0) * VE;
    const T* base = p - skip;
    float best = -INFINITY;
    auto take = [&](int u, float* x) {                                             // (NaN: as -inf, -0: as +0)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            x[e] = x[e] == x[e] ? x[e] + 0.f : -INFINITY;
            best = fmaxf(best, x[e]);
        }
#pragma unroll
        for (int e = 0; e < VE; e += 4) *reinterpret_cast<float4*>(x_s + u * VE + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
    };
    // whole vectors, four on their way at a time; the row's first and last one by elements
    const int whole0 = unit0 == 0 && skip > 0 ? 1 : 0, whole1 = n / VE - (unit0 + n / VE == units && end % VE != 0 ? 1 : 0);
    constexpr int BATCH = 4;
    for (int u0 = whole0 + tid; u0 < whole1; u0 += threads * BATCH) {
        uint4 raw[BATCH];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int u = u0 + e * threads;
            if (u < whole1) raw[e] = __ldg(reinterpret_cast<const uint4*>(base) + unit0 + u);
        }
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int u = u0 + e * threads;
            if (u >= whole1) break;
            float x[VE];
            Vec16<T>::unpack(raw[e], x);
            take(u, x);
        }
    }
    const int edge = tid == 0 && whole0 > 0 ? 0 : tid == 1 && whole1 < n / VE && (whole1 > 0 || whole0 == 0) ? whole1 : -1;
    if (edge >= 0) {
        const long long at = (long long)(unit0 + edge) * VE;
        float x[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            x[e] = -INFINITY;
            if (at + e >= skip && at + e < end) {
                if constexpr (sizeof(T) == 2) x[e] = __bfloat162float(base[at + e]);
                else x[e] = base[at + e];
            }
        }
        take(edge, x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    if ((tid & 31) == 0) warp_largest_s[tid >> 5] = best;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < threads / 32; ++w) best = fmaxf(best, warp_largest_s[w]);
        largest_s = best;
    }
    sync();
    Row r;
    r.largest = -INFINITY;
    for (int c = 0; c < ctas; ++c) r.largest = fmaxf(r.largest, *cluster.map_shared_rank(&largest_s, c));
    const float t = a.temperature ? a.temperature[row] : 1.f, u = a.uniforms[row];
    r.greedy = !(t > 0.f);
    const double inverse_t = 1.0 / (double)t;
    r.places = a.places;
    r.scale = inverse_t * (256.0 * 1.4426950408889634074);
    // 2^(F + 1) of them make one unit.  (Where that lies below every float, or T is infinite: only -inf has none.  Below +inf everything has none.)
    r.zero_from = isinf(r.largest) ? r.largest : fmaxf((float)((double)r.largest - (a.places + 1) * 0.69314718055994530942 * (double)t), -FLT_MAX);
    const int k = a.top_k ? a.top_k[row] : 0;
    const float top_p = a.top_p ? a.top_p[row] : 1.f, min_p_given = a.min_p ? a.min_p[row] : 0.f;
    const bool use_k = k >= 1 && k < a.vocab, use_p = top_p < 1.f;
    const double unit = (double)(1ull << a.places);
    const u64 least = min_p_given > 0.f ? (u64)ceil(fmin((double)min_p_given, 1.0) * unit) : 1;     // (at least one unit: what has none is never drawn)
    const bool nothing = r.largest == -INFINITY;

    // ---- a histogram of the slice's tokens, summed over the cluster into all_*[which] ----
    auto reduce = [&](bool fine, bool masses) {
        sync();
        const int share = (fine ? FINE : BINS) / ctas;
#pragma unroll 1
        for (int b = tid; b < share; b += threads) {
            const int at = rank * share + b;
            uint32_t count[MAX_CLUSTER], low[MAX_CLUSTER], high[MAX_CLUSTER];
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c) {
                count[c] = low[c] = high[c] = 0;
                if (c < ctas) {
                    const Histograms* h = cluster.map_shared_rank(hist, c);
                    count[c] = h->count[at];
                    if (masses) {
                        low[c] = h->low[at];
                        high[c] = h->high[at];
                    }
                }
            }
            uint32_t all = 0;
            u64 m = 0;
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c) {
                all += count[c];
                m += (u64)low[c] | (u64)high[c] << 32;
            }
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c)
                if (c < ctas) {
                    Histograms* h = cluster.map_shared_rank(hist, c);
                    (fine ? h->fine_count : h->all_count)[at] = all;
                    (fine ? h->fine_mass : h->all_mass)[at] = m;
                }
        }
        sync();
    };
    static_assert(BINS % MAX_CLUSTER == 0 && FINE % MAX_CLUSTER == 0, "shares");
    auto clear = [&] {
#pragma unroll 1
        for (int b = tid; b < BINS; b += threads) hist->count[b] = hist->low[b] = hist->high[b] = 0;
        __syncthreads();
    };
    auto add = [&](int b, u64 m, bool counts) {
        if (counts) atomicAdd(&hist->count[b], 1u);
        if (m == 0) return;
        const uint32_t low = (uint32_t)m, old = atomicAdd(&hist->low[b], low);
        const uint32_t high = (uint32_t)(m >> 32) + (old + low < old);
        if (high) atomicAdd(&hist->high[b], high);
    };
    // The bin (of the first or a finer histogram) in which the count passes `want` (by_mass: the mass reaches `target`), and what of either lies
    // before it.
    auto find = [&](bool fine, bool by_mass, uint32_t want, double target, u64 base0) {
        const int bins = fine ? FINE : BINS, per = (bins + threads - 1) / threads, at = tid * per;
        const uint32_t* counts = fine ? hist->fine_count : hist->all_count;
        const u64* masses = fine ? hist->fine_mass : hist->all_mass;
        u64 count = 0, m = 0, all;
#pragma unroll 1
        for (int b = at; b < min(bins, at + per); ++b) {
            count += counts[b];
            m += masses[b];
        }
        u64 before = base0 + block_exclusive_scan<u64>(by_mass ? m : count, scan64_s, &all);
#pragma unroll 1
        for (int b = at; b < min(bins, at + per); ++b) {
            const u64 step = by_mass ? masses[b] : counts[b];
            const bool here = by_mass ? (double)before < target && (double)(before + step) >= target : before < want && before + step >= want;
            if (here) {
                found_bin_s = b;
                found_count_s = counts[b];
                found_mass_s = masses[b];
                found_before_s = before;
            }
            before += step;
        }
        __syncthreads();
    };
    // All tokens of the slice, four at a time: a warp has a run of neighbours.  (What works on a token has no branches: four tokens hide each
    // other's latency.)
    const int lane = tid & 31, run4 = ((n / 4 + threads / 32 - 1) / (threads / 32) + 31) & ~31, first4 = (tid >> 5) * run4;      // in fours
    auto fours = [&](auto f) {
#pragma unroll 1
        for (int i = lane; i < run4; i += 32)
            f(first4 + i < n / 4 ? *reinterpret_cast<const float4*>(x_s + 4 * (first4 + i)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY));
    };
    auto each_token = [&](auto f) {
#pragma unroll 1
        for (int j = tid; j < n / 4; j += threads) {
            const float4 x = *reinterpret_cast<const float4*>(x_s + 4 * j);
            f(x.x);
            f(x.y);
            f(x.z);
            f(x.w);
        }
    };
    // ... but for those all of whose neighbours in the warp are below `from`
    auto each_token_from = [&](float from, auto f) {
        fours([&](float4 x) {
            if (!__any_sync(0xffffffffu, fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)) >= from)) return;
            f(x.x);
            f(x.y);
            f(x.z);
            f(x.w);
        });
    };
    // Four sums over the threads of the whole cluster, in row_part_s
    int flip = 0;
    auto sum_over_row = [&](u64 v0, u64 v1, u64 v2, u64 v3) {
        u64 v[4] = {v0, v1, v2, v3};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], o);
            if ((tid & 31) == 0) part_s[tid >> 5][e] = v[e];
        }
        __syncthreads();
        if (tid < 4) {
            u64 x = 0;
            for (int w = 0; w < threads / 32; ++w) x += part_s[w][tid];
            cta_part_s[flip][tid] = x;
        }
        sync();
        if (tid < 32) {                                                            // lane: CTA tid / 4, sum tid % 4
            u64 x = (tid >> 2) < ctas ? *cluster.map_shared_rank(&cta_part_s[flip][tid & 3], tid >> 2) : 0;
#pragma unroll
            for (int o = 16; o > 2; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (tid < 4) row_part_s[tid] = x;
        }
        __syncthreads();
        flip ^= 1;
    };
    // From bin `bin` of the first histogram, which holds `count` tokens, down to the end of the run: towards `want` tokens (by_mass: a mass of
    // `target`), `before` of them (of it) in the bins above.
    auto descend = [&](int bin, uint32_t count, bool by_mass, uint32_t want, double target, u64 before, u64 m) {
        Cut c{bin, bin_from(r, bin), bin_to(r, bin), 0u, 0u, 0u};
        c.low = key_of<T>(c.from);
        c.high = key_of<T>(c.to);
        bool counted = use_k;                                                      // (the first histogram counts for top-k only)
        while (!counted || (count > 1 && c.low != c.high)) {
            counted = true;
            const uint32_t range = c.high - c.low;                                 // bins of 2^shift keys, from the largest down
            const int shift = range < FINE ? 0 : 32 - __clz(range) - 9;
            clear();
            fours([&](float4 x4) {
                const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool near = x[e] >= c.from && x[e] <= c.to;
                    if (!__any_sync(0xffffffffu, near)) continue;
                    const uint32_t key = key_of<T>(x[e]);
                    if (near && key - c.low <= range && first_bin(r, x[e]) == c.bin) add((int)((c.high - key) >> shift), by_mass ? mass(r, table_s, x[e]) : 0, true);
                }
            });
            reduce(true, by_mass);
            find(true, by_mass, want, target, before);
            const uint32_t top = c.high - ((uint32_t)found_bin_s << shift), span = (1u << shift) - 1;
            c.low = top - c.low > span ? top - span : c.low;
            c.high = top;
            count = found_count_s;
            before = found_before_s;
            m = found_mass_s;
            __syncthreads();                                                       // found_* may be written again
        }
        if (by_mass) {
            const u64 one = m / count;                                             // tokens of one value have one mass
            uint32_t low = 1, high = count;                                        // the fewest that reach the target
            while (low < high) {
                const uint32_t mid = low + (high - low) / 2;
                if ((double)(before + mid * one) >= target) high = mid;
                else low = mid + 1;
            }
            c.ties = low;
        } else {
            c.ties = want - (uint32_t)before;
        }
        return c;
    };

    Cut cut{-1, 0.f, 0.f, 0u, 0u, 0u};
    if (!nothing && !r.greedy && (use_k || use_p)) {
        clear();
        if (use_p) each_token([&](float x) { add(first_bin(r, x), mass(r, table_s, x), use_k); });
        else each_token([&](float x) { atomicAdd(&hist->count[first_bin(r, x)], 1u); });
        reduce(false, use_p);
        u64 kept;
        auto found = [&](bool by_mass, uint32_t want, double target) {
            const int bin = found_bin_s;
            const uint32_t count = found_count_s;
            const u64 before = found_before_s, m = found_mass_s;
            __syncthreads();
            return descend(bin, count, by_mass, want, target, before, m);
        };
        if (use_k) {
            find(false, false, (uint32_t)k, 0.0, 0);
            cut = found(false, (uint32_t)k, 0.0);
        }
        if (use_p) {
            u64 part = 0, tie = 0;                                                 // the mass of what is kept so far
            uint32_t tie_tokens = 0;
            for (int b = tid; b < BINS; b += threads)
                if (!use_k || b < cut.bin) part += hist->all_mass[b];
            if (use_k) {
                part = rank == 0 ? part : 0;
                fours([&](float4 x4) {
                    const float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool near = x[e] >= cut.from && x[e] <= cut.to;
                        if (!__any_sync(0xffffffffu, near)) continue;
                        const int s = near && first_bin(r, x[e]) == cut.bin ? side<T>(r, cut, x[e]) : -1;
                        const u64 m = mass(r, table_s, x[e]);
                        part += s > 0 ? m : 0;
                        tie += s == 0 ? m : 0;
                        tie_tokens += s == 0;
                    }
                });
                sum_over_row(part, tie, tie_tokens, 0);
                kept = row_part_s[0] + (row_part_s[2] ? row_part_s[1] / row_part_s[2] * cut.ties : 0);
            } else {
                block_exclusive_scan<u64>(part, scan64_s, &kept);
                __syncthreads();
            }
            const double target = fmax((double)top_p * (double)kept, 0.5);         // (the largest is always kept)
            find(false, true, 0u, target, 0);
            cut = found(true, 0u, target);
        }
    }

    // ---- the draw: kept masses by warps (runs of neighbours), then the one run that passes the target token by token ----
    // (a quick no for most: what lies below the cut's bin, or has no mass, or clearly less than min-p)
    float floor_x = r.zero_from;
    if (cut.bin >= 0) floor_x = fmaxf(floor_x, cut.from);
    if (min_p_given > 0.f && t < INFINITY) floor_x = fmaxf(floor_x, (float)((double)r.largest + (double)t * (log(fmin((double)min_p_given, 1.0)) - 1e-3)) - fabsf(r.largest) * 0x1p-22f);
    if (r.greedy) floor_x = r.largest;
    // 1: kept, 0: a tie at the end of the run, -1: not kept; its mass, 0 where not kept
    auto kept_side = [&](float x, u64* m) {
        int s = r.greedy ? (x == r.largest ? 0 : -1) : side<T>(r, cut, x);
        *m = mass(r, table_s, x);
        s = *m >= least ? s : -1;
        *m = s >= 0 ? *m : 0;
        return s;
    };
    const uint32_t ties = r.greedy ? 1u : cut.ties;
    u64 sum = 0, tie_mass = 0;
    uint32_t tie_count = 0;
    auto tally = [&](float x) {
        u64 m;
        const int s = kept_side(x, &m);
        sum += s > 0 ? m : 0;
        tie_count += s == 0;
        tie_mass = s == 0 ? m : tie_mass;
    };
    if (!nothing) {
        if (cut.bin < 0 && !r.greedy)
            each_token_from(floor_x, [&](float x) {
                const u64 m = mass(r, table_s, x);
                sum += m >= least ? m : 0;
            });
        else if (r.greedy)
            each_token_from(floor_x, tally);
        else
            fours([&](float4 x4) {
                const float x[4] = {x4.x, x4.y, x4.z, x4.w};
                if (!__any_sync(0xffffffffu, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= floor_x)) return;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u64 m = mass(r, table_s, x[e]);
                    sum += x[e] > cut.to && m >= least ? m : 0;                    // above the cut's bin
                    const bool near = x[e] >= cut.from && x[e] <= cut.to;
                    if (__any_sync(0xffffffffu, near) && near) tally(x[e]);
                }
            });
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        tie_count += __shfl_xor_sync(0xffffffffu, tie_count, o);
        tie_mass = max(tie_mass, __shfl_xor_sync(0xffffffffu, tie_mass, o));
    }
    if (lane == 0) {
        run_sum_s[tid >> 5] = sum;
        run_ties_s[tid >> 5] = tie_count;
        run_tie_mass_s[tid >> 5] = tie_mass;
    }
    __syncthreads();
    if (tid < 32) {                                                                // what lies before each run; the CTA's totals
        u64 m = lane < threads / 32 ? run_sum_s[lane] : 0, before = m;
        uint32_t c = lane < threads / 32 ? run_ties_s[lane] : 0, ties_before = c;
        u64 one = lane < threads / 32 ? run_tie_mass_s[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 y = __shfl_up_sync(0xffffffffu, before, o);
            const uint32_t z = __shfl_up_sync(0xffffffffu, ties_before, o);
            if (lane >= o) {
                before += y;
                ties_before += z;
            }
            one = max(one, __shfl_xor_sync(0xffffffffu, one, o));
        }
        run_sum_s[lane] = before - m;
        run_ties_s[lane] = ties_before - c;
        if (lane == 31) {
            total_mass_s = before;
            total_ties_s = ties_before;
            tie_mass_s = one;
            run_found_s = -1;
        }
    }
    sync();
    u64 total = 0, cta_before = 0;
    uint32_t all_ties = 0, cta_ties_before = 0;
    tie_mass = 0;
#pragma unroll
    for (int c = 0; c < MAX_CLUSTER; ++c) {
        if (c == rank) {
            cta_before = total;
            cta_ties_before = all_ties;
        }
        if (c < ctas) {
            total += *cluster.map_shared_rank(&total_mass_s, c);
            all_ties += *cluster.map_shared_rank(&total_ties_s, c);
            tie_mass = max(tie_mass, *cluster.map_shared_rank(&tie_mass_s, c));
        }
    }
    auto running = [&](u64 m, uint32_t t) { return m + min(t, ties) * tie_mass; };
    const u64 whole = running(total, all_ties);
    if (nothing || whole == 0) {
        if (rank == 0 && tid == 0) {
            a.tokens[row] = -1;
            if (a.logprobs) a.logprobs[row] = -INFINITY;
        }
    } else {
        const double wanted = floor((u > 0.f ? fmin((double)u, 1.0) : 0.0) * (double)whole);
        const u64 target = min((u64)wanted, whole - 1);
        const u64 m0 = cta_before + run_sum_s[tid >> 5], m1 = cta_before + ((tid >> 5) + 1 < threads / 32 ? run_sum_s[(tid >> 5) + 1] : total_mass_s);
        const uint32_t t0 = cta_ties_before + run_ties_s[tid >> 5], t1 = cta_ties_before + ((tid >> 5) + 1 < threads / 32 ? run_ties_s[(tid >> 5) + 1] : total_ties_s);
        if (lane == 0 && running(m0, t0) <= target && target < running(m1, t1)) run_found_s = tid >> 5;
        __syncthreads();
        const int run = run_found_s;
        if (run >= 0) {                                                            // (the whole CTA: a few neighbours per thread)
            const int per = (run4 * 4 + threads - 1) / threads, begin = run * run4 * 4 + tid * per, stop = min(n, min(begin + per, (run + 1) * run4 * 4));
            u64 mine = 0, all;
            uint32_t my_ties = 0, all_run_ties;
#pragma unroll 1
            for (int j = begin; j < stop; ++j) {
                u64 m;
                const int s = kept_side(x_s[j], &m);
                mine += s > 0 ? m : 0;
                my_ties += s == 0;
            }
            u64 at = cta_before + run_sum_s[run] + block_exclusive_scan<u64>(mine, scan64_s, &all);
            uint32_t tie_at = cta_ties_before + run_ties_s[run] + block_exclusive_scan<uint32_t>(my_ties, scan32_s, &all_run_ties);
            if (running(at, tie_at) <= target && target < running(at + mine, tie_at + my_ties)) {
#pragma unroll 1
                for (int j = begin; j < stop; ++j) {
                    u64 m;
                    const int s = kept_side(x_s[j], &m);
                    at += s > 0 ? m : 0;
                    tie_at += s == 0;
                    if (target < running(at, tie_at)) {
                        a.tokens[row] = (int32_t)((long long)unit0 * VE + j - skip);
                        if (a.logprobs)
                            a.logprobs[row] = r.greedy ? 0.f : (float)((x_s[j] == r.largest ? 0.0 : ((double)x_s[j] - (double)r.largest) * inverse_t) - log((double)whole / unit));
                        break;
                    }
                }
            }
        }
    }
    if (ctas > 1) cluster.sync();                                                  // nobody leaves while others read its memory
}

template <typename T>
cudaError_t launch_sample(SampleArgs a, int rows, cudaStream_t stream) {
    constexpr int VE = 16 / (int)sizeof(T), MAX_DEVICES = 64;
    auto kern = sample_kernel<T>;
    static std::mutex setup_mutex;
    static bool ready[MAX_DEVICES] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(setup_mutex);
        if (!ready[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SLICE * 4 + (int)sizeof(Histograms));
            if (e != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    // CTAs per row: what its slices need, and more while the launch leaves SMs idle and a slice is worth a CTA
    const int units = a.vocab / VE + 2;                                            // (a row may start and end inside a vector)
    int ctas = 1;
    while (ctas < MAX_CLUSTER && (units + ctas - 1) / ctas * VE > MAX_SLICE) ctas *= 2;
    while (ctas < MAX_CLUSTER && (long long)rows * ctas * 2 <= 148 && a.vocab / ctas > 4096) ctas *= 2;
    const size_t smem = (size_t)((units + ctas - 1) / ctas) * VE * 4 + (a.histograms ? sizeof(Histograms) : 0);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * ctas));
    cfg.blockDim = dim3(a.vocab / ctas > 16384 ? 1024 : a.vocab / ctas > 4096 ? 512 : 128);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace
}  // namespace onela

extern "C" onela_status onela_sample_tokens(const onela_sample_args* g, void* stream) {
    using namespace onela;
    if (!g) return ONELA_E_INVAL;
    if (g->dtype != ONELA_DTYPE_F32 && g->dtype != ONELA_DTYPE_BF16) return ONELA_E_INVAL;
    if (g->rows < 0 || g->vocab < 1) return ONELA_E_INVAL;
    static_assert(MAX_VOCAB / 8 + 32 <= MAX_SLICE, "a slice with its row's odd start and end");
    if (g->vocab > MAX_VOCAB || g->rows > 0x7fffffff / MAX_CLUSTER) return ONELA_E_CAPACITY;
    if (g->rows == 0) return ONELA_OK;
    if (!g->logits_dev || !g->uniforms_dev || !g->tokens_out_dev || (g->logits_stride != 0 && g->logits_stride < g->vocab)) return ONELA_E_INVAL;
    if (reinterpret_cast<uintptr_t>(g->logits_dev) % (g->dtype == ONELA_DTYPE_BF16 ? 2 : 4) != 0) return ONELA_E_INVAL;
    if (!aligned4(g->uniforms_dev, g->temperature_dev, g->top_p_dev, g->min_p_dev, g->top_k_dev, g->tokens_out_dev, g->logprobs_out_dev)) return ONELA_E_INVAL;
    int log_vocab = 0;
    while ((1ll << log_vocab) < g->vocab) ++log_vocab;
    const SampleArgs a{g->logits_dev, g->uniforms_dev, g->temperature_dev, g->top_p_dev, g->min_p_dev, g->top_k_dev, g->tokens_out_dev, g->logprobs_out_dev,
                       g->logits_stride, g->vocab, 62 - log_vocab, g->top_k_dev != nullptr || g->top_p_dev != nullptr};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = g->dtype == ONELA_DTYPE_BF16 ? launch_sample<__nv_bfloat16>(a, g->rows, s) : launch_sample<float>(a, g->rows, s);
    return e == cudaSuccess ? ONELA_OK : ONELA_E_CUDA;
}
