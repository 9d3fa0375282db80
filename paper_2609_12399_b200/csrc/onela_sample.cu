// One token per row of logits, drawn with the caller's random numbers (onela_sample_tokens).
//
// With w_i = exp((x_i - max) / T) and the tokens ordered by (x descending, index ascending), top-k, top-p and min-p each keep a
// leading run of that order, so all of them together keep a leading run too, and no sort is needed: what is kept is everything above one
// value, and the first m (by index) of the tokens that have that value.  The token is where the running sum of the kept masses, in the order of
// indices, passes uniform * sum.
//
// A row lies in the shared memory of one cluster of 1 to 8 CTAs, read from memory once.  Masses are integers, w in units of 2^-F with F = 62 -
// ceil(log2 vocab) (43 places or more), so sums are exact in any order, atomics included.  w = 2^(n / 256 + f / 256) in 64 bits, |f| <= 1 / 2:
// 2^(n mod 256 / 256) from a table, the rest by its series to the third power (Tang 1989; relative error 2e-13): a third of the instructions of exp().
//   top-k   tokens counted by bins of their distance from the largest (1024 bins); the bin in which the count passes k is cut
//           into 1024 bins of the values' bit patterns, and so on until a bin holds one token or one value
//   top-p   the same descent on the bins' masses, from the same first histogram, towards top_p times the mass of the top-k tokens
// A histogram is reduced by the cluster (a CTA sums a share of the bins over all CTAs and hands the sums to all), two cluster barriers.
// What bounds it: launches of a few rows the chain of barriers, many rows the exponentials' and the histogram's instructions.
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

constexpr int MAX_THREADS = 1024, TABLE = 256, BINS = 1024, MAX_SLICE = 45056, MAX_CLUSTER = 8, MAX_VOCAB = 360000;
constexpr float BINS_PER_UNIT = 32.f;            // first histogram: bins of 1 / 32 up to 32 below the largest, the rest in the last one

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

struct Histograms {                              // of one round, and what the cluster made of the first and of the current one
    uint32_t count[BINS], low[BINS], high[BINS];
    uint32_t all_count[2][BINS];
    u64 all_mass[2][BINS];
};

// What every CTA of a row knows.
struct Row {
    float largest, zero_from;                    // what lies below zero_from has no mass
    double scale, offset;                        // 256 log2(e) / T, and the same times - largest
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
    const double y = fma((double)x, r.scale, r.offset), t = y + MAGIC, f = (y - (t - MAGIC)) * LN2;
    const int n = __double2loint(t);
    const double w = table[n & (TABLE - 1)], v = fma(w, f * fma(f, fma(f, 1.0 / 6.0, 0.5), 1.0), w);
    const u64 m = __double2ull_rn(__hiloint2double(__double2hiint(v) + ((n >> 8) + r.places) * (1 << 20), __double2loint(v)));
    return x == r.largest ? 1ull << r.places : x < r.zero_from ? 0 : m;
}

// The end of the kept run: tokens of first bin `bin` whose keys lie in [low, high] are its last ones, `ties` of them (by index) kept; what
// lies above is kept whole.
struct Cut {
    int bin;                                     // -1: everything is above
    uint32_t low, high, ties;
};
// 1 above, 0 at the end of the run, -1 below
template <typename T>
__device__ __forceinline__ int side(const Row& r, const Cut& c, float x) {
    if (c.bin < 0) return 1;
    const int b = first_bin(r, x);
    if (b != c.bin) return b < c.bin ? 1 : -1;
    const uint32_t k = key_of<T>(x);
    return k > c.high ? 1 : k >= c.low ? 0 : -1;
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
    __shared__ uint32_t total_ties_s;
    __shared__ int found_bin_s;
    __shared__ u64 found_mass_s, found_before_count_s, found_before_mass_s;
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
#pragma unroll 4
    for (int u = tid; u < n / VE; u += threads) {
        const long long at = (long long)(unit0 + u) * VE;
        float x[VE];
        if (at >= skip && at + VE <= end) {
            Vec16<T>::load(base + at, x);
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                x[e] = -INFINITY;
                if (at + e >= skip && at + e < end) {
                    if constexpr (sizeof(T) == 2) x[e] = __bfloat162float(base[at + e]);
                    else x[e] = base[at + e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            x[e] = x[e] == x[e] ? x[e] + 0.f : -INFINITY;
            best = fmaxf(best, x[e]);
        }
#pragma unroll
        for (int e = 0; e < VE; e += 4) *reinterpret_cast<float4*>(x_s + u * VE + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
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
    const float t = a.temperature ? a.temperature[row] : 1.f;
    r.greedy = !(t > 0.f);
    const double inverse_t = 1.0 / (double)t;
    r.places = a.places;
    r.scale = inverse_t * (256.0 * 1.4426950408889634074);
    r.offset = -(double)r.largest * r.scale;
    // 2^(F + 1) of them make one unit.  (Where that lies below every float, or T is infinite: only -inf has none.)
    r.zero_from = fmaxf((float)((double)r.largest - (a.places + 1) * 0.69314718055994530942 * (double)t), -FLT_MAX);
    const int k = a.top_k ? a.top_k[row] : 0;
    const float top_p = a.top_p ? a.top_p[row] : 1.f, min_p_given = a.min_p ? a.min_p[row] : 0.f;
    const bool use_k = k >= 1 && k < a.vocab, use_p = top_p < 1.f;
    const double unit = (double)(1ull << a.places);
    const u64 least = min_p_given > 0.f ? (u64)ceil(fmin((double)min_p_given, 1.0) * unit) : 1;     // (at least one unit: what has none is never drawn)
    const bool nothing = r.largest == -INFINITY;

    // ---- a histogram of the slice's tokens, summed over the cluster into all_*[which] ----
    auto reduce = [&](int which) {
        sync();
        const int share = BINS / ctas;
        for (int b = tid; b < share; b += threads) {
            const int at = rank * share + b;
            uint32_t count = 0;
            u64 m = 0;
            for (int c = 0; c < ctas; ++c) {
                const Histograms* h = cluster.map_shared_rank(hist, c);
                count += h->count[at];
                m += (u64)h->low[at] | (u64)h->high[at] << 32;
            }
            for (int c = 0; c < ctas; ++c) {
                Histograms* h = cluster.map_shared_rank(hist, c);
                h->all_count[which][at] = count;
                h->all_mass[which][at] = m;
            }
        }
        sync();
    };
    auto clear = [&] {
        for (int b = tid; b < BINS; b += threads) hist->count[b] = hist->low[b] = hist->high[b] = 0;
        __syncthreads();
    };
    auto add = [&](int b, float x, bool counts, bool masses) {
        if (counts) atomicAdd(&hist->count[b], 1u);
        if (!masses) return;
        const u64 m = mass(r, table_s, x);
        if (m == 0) return;
        const uint32_t low = (uint32_t)m, old = atomicAdd(&hist->low[b], low);
        const uint32_t high = (uint32_t)(m >> 32) + (old + low < old);
        if (high) atomicAdd(&hist->high[b], high);
    };
    // The bin of all_*[which] in which the count passes `want` (by_mass: the mass reaches `target`), and what lies before it (of the mass
    // only where masses are kept, of the count only where it is what is looked for).
    auto find = [&](int which, bool by_mass, bool masses, uint32_t want, double target, u64 count0, u64 mass0) {
        const int per = BINS / threads, at = tid * per;
        u64 count = 0, m = 0, all;
        for (int b = 0; b < per; ++b) {
            count += hist->all_count[which][at + b];
            m += hist->all_mass[which][at + b];
        }
        u64 before = by_mass ? 0 : count0 + block_exclusive_scan<u64>(count, scan64_s, &all);
        u64 mass_before = masses ? mass0 + block_exclusive_scan<u64>(m, scan64_s, &all) : 0;
        for (int b = 0; b < per; ++b) {
            const u64 w = hist->all_mass[which][at + b];
            const uint32_t c = hist->all_count[which][at + b];
            const bool here = by_mass ? (double)mass_before < target && (double)(mass_before + w) >= target : before < want && before + c >= want;
            if (here) {
                found_bin_s = at + b;
                found_count_s = c;
                found_mass_s = w;
                found_before_count_s = before;
                found_before_mass_s = mass_before;
            }
            before += c;
            mass_before += w;
        }
        __syncthreads();
    };
    // all tokens of the slice, four at a time
    auto each_token = [&](auto f) {
        for (int j = tid; j < n / 4; j += threads) {
            const float4 x = *reinterpret_cast<const float4*>(x_s + 4 * j);
            f(x.x);
            f(x.y);
            f(x.z);
            f(x.w);
        }
    };
    // From the first histogram (all_*[0]) down to the end of the run; *kept_mass: the run's mass (with masses).
    auto descend = [&](bool by_mass, uint32_t want, double target, bool masses, u64* kept_mass) {
        find(0, by_mass, masses, want, target, 0, 0);
        Cut c{found_bin_s, 0u, key_of<T>(INFINITY), 0u};
        // keys that the bin can hold, half a bin more on either side (the bin of a value is off by far less)
        if (c.bin < BINS - 1) {
            c.low = key_of<T>((float)((double)r.largest - (c.bin + 1.5) / BINS_PER_UNIT));
            c.high = key_of<T>((float)((double)r.largest - (c.bin - 0.5) / BINS_PER_UNIT));
        } else {
            c.high = key_of<T>((float)((double)r.largest - (c.bin - 0.5) / BINS_PER_UNIT));
        }
        if (isinf(r.largest)) {
            c.low = 0u;
            c.high = key_of<T>(INFINITY);
        }
        uint32_t count = found_count_s;
        bool counted = use_k;                                                      // (the first histogram counts for top-k only)
        u64 m = found_mass_s, before = found_before_count_s, mass_before = found_before_mass_s;
        while (!counted || (count > 1 && c.low != c.high)) {
            counted = true;
            const uint32_t range = c.high - c.low;                                 // bins of 2^shift keys, from the largest down
            const int shift = range < BINS ? 0 : 32 - __clz(range) - 10;
            clear();
            each_token([&](float x) {
                const uint32_t key = key_of<T>(x);
                if (key - c.low <= range && first_bin(r, x) == c.bin) add((int)((c.high - key) >> shift), x, true, masses);
            });
            reduce(1);
            find(1, by_mass, masses, want, target, before, mass_before);
            const uint32_t top = c.high - ((uint32_t)found_bin_s << shift), span = (1u << shift) - 1;
            c.low = top - c.low > span ? top - span : c.low;
            c.high = top;
            count = found_count_s;
            before = found_before_count_s;
            m = found_mass_s;
            mass_before = found_before_mass_s;
            __syncthreads();                                                       // found_* may be written again
        }
        const u64 one = count ? m / count : 0;                                     // tokens of one value have one mass
        if (by_mass) {
            uint32_t low = 1, high = max(count, 1u);                               // the fewest that reach the target
            while (low < high) {
                const uint32_t mid = low + (high - low) / 2;
                if ((double)(mass_before + mid * one) >= target) high = mid;
                else low = mid + 1;
            }
            c.ties = low;
        } else {
            c.ties = want - (uint32_t)before;
        }
        *kept_mass = mass_before + c.ties * one;
        return c;
    };

    Cut cut{-1, 0u, 0u, 0u};
    if (!nothing && !r.greedy && (use_k || use_p)) {
        clear();
        if (use_p) each_token([&](float x) { add(first_bin(r, x), x, use_k, true); });
        else each_token([&](float x) { add(first_bin(r, x), x, true, false); });
        reduce(0);
        u64 kept = 0;
        if (use_k) {
            cut = descend(false, (uint32_t)k, 0.0, use_p, &kept);
        } else {
            u64 part = 0;
            for (int b = tid; b < BINS; b += threads) part += hist->all_mass[0][b];
            block_exclusive_scan<u64>(part, scan64_s, &kept);
        }
        if (use_p) {
            __syncthreads();
            const double target = fmax((double)top_p * (double)kept, 0.5);         // (the largest is always kept)
            cut = descend(true, 0u, target, true, &kept);
        }
    }

    // ---- the draw: thread = L consecutive tokens (L odd: no bank conflicts) ----
    const int L = ((n + threads - 1) / threads) | 1, begin = min(n, tid * L), stop = min(n, begin + L);
    auto kept_side = [&](float x, u64* m) {                                        // side() with min-p, and the mass
        const int s = r.greedy ? (x == r.largest ? 0 : -1) : side<T>(r, cut, x);
        if (s < 0) return -1;
        *m = mass(r, table_s, x);
        return *m >= least ? s : -1;
    };
    const uint32_t ties = r.greedy ? 1u : cut.ties;
    u64 sum = 0, tie_mass = 0;
    uint32_t tie_count = 0;
    if (!nothing) {
        for (int j = begin; j < stop; ++j) {
            u64 m;
            const int s = kept_side(x_s[j], &m);
            if (s > 0) sum += m;
            else if (s == 0) {
                ++tie_count;
                tie_mass = m;
            }
        }
    }
    u64 cta_sum;
    uint32_t cta_ties;
    const u64 sum_before = block_exclusive_scan<u64>(sum, scan64_s, &cta_sum);
    const uint32_t ties_before = block_exclusive_scan<uint32_t>(tie_count, scan32_s, &cta_ties);
    if (tid == 0) {
        total_mass_s = cta_sum;
        total_ties_s = cta_ties;
        tie_mass_s = 0;
    }
    __syncthreads();
    if (tie_count) tie_mass_s = tie_mass;                                          // (the same from every thread)
    sync();
    u64 total = 0, cta_before = 0;
    uint32_t all_ties = 0, cta_ties_before = 0;
    tie_mass = 0;
    for (int c = 0; c < ctas; ++c) {
        if (c == rank) {
            cta_before = total;
            cta_ties_before = all_ties;
        }
        total += *cluster.map_shared_rank(&total_mass_s, c);
        all_ties += *cluster.map_shared_rank(&total_ties_s, c);
        tie_mass = max(tie_mass, *cluster.map_shared_rank(&tie_mass_s, c));
    }
    auto running = [&](u64 m, uint32_t t) { return m + min(t, ties) * tie_mass; };
    const u64 whole = running(total, all_ties);
    if (nothing || whole == 0) {
        if (rank == 0 && tid == 0) {
            a.tokens[row] = -1;
            if (a.logprobs) a.logprobs[row] = -INFINITY;
        }
    } else {
        const float u = a.uniforms[row];
        const double wanted = floor((u > 0.f ? fmin((double)u, 1.0) : 0.0) * (double)whole);
        const u64 target = min((u64)wanted, whole - 1);
        u64 m0 = cta_before + sum_before;
        uint32_t t0 = cta_ties_before + ties_before;
        const uint32_t here = __ballot_sync(0xffffffffu, running(m0, t0) <= target && target < running(m0 + sum, t0 + tie_count));
        if (here) {                                                                // the warp goes through the one thread's tokens
            const int lane = tid & 31, owner = __ffs(here) - 1;
            m0 = __shfl_sync(0xffffffffu, m0, owner);
            t0 = __shfl_sync(0xffffffffu, t0, owner);
            const int first = __shfl_sync(0xffffffffu, begin, owner), last = __shfl_sync(0xffffffffu, stop, owner);
            for (int j0 = first; j0 < last; j0 += 32) {
                const int j = j0 + lane;
                u64 m = 0;
                const int s = j < last ? kept_side(x_s[j], &m) : -1;
                u64 run = s > 0 ? m : 0;
                uint32_t count = s == 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 y = __shfl_up_sync(0xffffffffu, run, o);
                    const uint32_t c = __shfl_up_sync(0xffffffffu, count, o);
                    if (lane >= o) {
                        run += y;
                        count += c;
                    }
                }
                const uint32_t past = __ballot_sync(0xffffffffu, target < running(m0 + run, t0 + count));
                if (past) {
                    if (lane == __ffs(past) - 1) {
                        a.tokens[row] = (int32_t)((long long)unit0 * VE + j - skip);
                        if (a.logprobs)
                            a.logprobs[row] = r.greedy ? 0.f : (float)((x_s[j] == r.largest ? 0.0 : ((double)x_s[j] - (double)r.largest) * inverse_t) - log((double)whole / unit));
                    }
                    break;
                }
                m0 += __shfl_sync(0xffffffffu, run, 31);
                t0 += __shfl_sync(0xffffffffu, count, 31);
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
    if (!g->logits_dev || !g->uniforms_dev || !g->tokens_out_dev || g->logits_stride < g->vocab) return ONELA_E_INVAL;
    if (reinterpret_cast<uintptr_t>(g->logits_dev) % (g->dtype == ONELA_DTYPE_BF16 ? 2 : 4) != 0) return ONELA_E_INVAL;
    int log_vocab = 0;
    while ((1ll << log_vocab) < g->vocab) ++log_vocab;
    const SampleArgs a{g->logits_dev, g->uniforms_dev, g->temperature_dev, g->top_p_dev, g->min_p_dev, g->top_k_dev, g->tokens_out_dev, g->logprobs_out_dev,
                       g->logits_stride, g->vocab, 62 - log_vocab, g->top_k_dev != nullptr || g->top_p_dev != nullptr};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = g->dtype == ONELA_DTYPE_BF16 ? launch_sample<__nv_bfloat16>(a, g->rows, s) : launch_sample<float>(a, g->rows, s);
    return e == cudaSuccess ? ONELA_OK : ONELA_E_CUDA;
}
