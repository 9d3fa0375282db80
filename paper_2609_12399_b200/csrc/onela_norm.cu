// Norms of queries and keys for each head with the rotation by position in the same pass (onela_norm_rotate).
//
// A head vector x of d elements becomes y = x / sqrt(sum x^2 + eps) or x / sqrt(mean x^2 + eps) * w, its first r elements turn in pairs
// by the angle position * inv_freq[i], queries are scaled.  Every element is read once and written once, so HBM bounds it.
//
// A row is one (token, head); 4 to 32 lanes share it, one or two pieces of 8 elements (16 bytes of bf16, 32 of fp32) each, and a thread has four
// pieces in flight.
// A CTA takes a few whole tokens, queries' and keys' heads alike: as many as leave the fewest passes of rows one after
// another (18 heads of 256 in passes of 32 rows: 7 tokens fill 126 of the rows of four passes, one token would leave 14 of 32 idle).  The angles belong to the token:
// cosine and sine are formed once per CTA, in shared memory.  position * inv_freq is exact in 64 bits (31 + 24 bits; two more than fit are
// rounded), reduced there to a fraction of a turn, and only the fraction goes through the fp32 functions, so far positions lose nothing.
// Measured: 16 384 tokens x 64 heads of 128 80.5 us (6.7 TB/s, the copy's rate; one piece per lane 92, 64-bit row numbers and a division per row
// 153, the next pass's rows ahead of this one's work 109), 4099 tokens x 18 heads of 256 with weights and rotation out of a projection's rows 17.3 us (issue
// slots; one piece per lane 27.6).
// Elements i and i + r / 2 lie in different lanes of a row (r is a multiple of 16), 8 shuffles away.
#include <algorithm>
#include <cmath>

#include "onela_internal.h"
#include "onela_layout.cuh"

namespace onela {
namespace {

constexpr int THREADS = 256, ROWS_IN_FLIGHT = 4, OCCUPANCY = 4;

struct NormArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const float *q_weight, *k_weight;
    const int32_t* positions;
    const float* inv_freq;
    long long q_stride, k_stride, q_out_stride, k_out_stride, n_tokens;
    int32_t hq, heads, dim, rotary, interleaved, norm;
    float eps, q_scale, sum_weight;                         // sum_weight: of the sum of squares beside eps
    int32_t tokens;                                         // of a CTA
    uint32_t magic;                                         // of a division by `heads`
};

template <typename T>
struct Raw {                                            // 8 elements as they lie in memory
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int c = 0; c < (int)sizeof(T) / 2; ++c) w[c] = __ldg(reinterpret_cast<const uint4*>(p) + c);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int c = 0; c < (int)sizeof(T) / 2; ++c) w[c] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void unpack(float2* x) const {
        float y[8];
#pragma unroll
        for (int c = 0; c < (int)sizeof(T) / 2; ++c) Vec16<T>::unpack(w[c], y + c * Vec16<T>::N);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = make_float2(y[2 * e], y[2 * e + 1]);
    }
};
enum { NO_ROTATION, HALVES, INTERLEAVED };

// LPR lanes per row, CHUNKS pieces of 8 elements per lane (piece c of lane l: elements 8 (c LPR + l) ..)
template <typename T, int LPR, int CHUNKS, int ROTATION>
__global__ void __launch_bounds__(THREADS, OCCUPANCY) norm_rotate_kernel(const NormArgs a) {
    constexpr int GROUPS = THREADS / LPR, ROWS = ROWS_IN_FLIGHT / CHUNKS, TILE = GROUPS * ROWS;
    extern __shared__ __align__(16) float turn_s[];         // [tokens of the CTA][cos r / 2 | sin r / 2 | -sin r / 2]
    __shared__ __align__(16) float weight_s[2][256];
    const int half = a.rotary / 2, lane = threadIdx.x % LPR, group = threadIdx.x / LPR, at = lane * 8;
    const long long token0 = (long long)blockIdx.x * a.tokens;
    const int tokens = (int)min((long long)a.tokens, a.n_tokens - token0), rows = tokens * a.heads;
    const T *q = static_cast<const T*>(a.q) + token0 * a.q_stride + at, *k = static_cast<const T*>(a.k) + token0 * a.k_stride + at;
    T *q_out = static_cast<T*>(a.q_out) + token0 * a.q_out_stride + at, *k_out = static_cast<T*>(a.k_out) + token0 * a.k_out_stride + at;
    const bool weights = a.q_weight || a.k_weight;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // (a CTA's tokens lie within 2^31 elements: launch_shape)
    const int q_step = (int)a.q_stride, k_step = (int)a.k_stride, q_out_step = (int)a.q_out_stride, k_out_step = (int)a.k_out_stride;
    auto token_of = [&](int row) { return (int)__umulhi((uint32_t)row, a.magic); };
    for (int base = 0; base < rows; base += TILE) {
        Raw<T> raw[ROWS][CHUNKS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = base + i * GROUPS + group, tok = token_of(row), head = row - tok * a.heads;
            const bool is_q = head < a.hq;
            const T* p = (is_q ? q : k) + (tok * (is_q ? q_step : k_step) + (is_q ? head : head - a.hq) * a.dim);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (row < rows && at + c * (LPR * 8) < a.dim) raw[i][c].load(p + c * (LPR * 8));
                else raw[i][c].clear();
            }
        }
        if (base == 0) {
            if (weights) {                                  // with the queries' scale in theirs (a rotation passes it on)
                for (int e = threadIdx.x; e < a.dim; e += THREADS) {
                    weight_s[0][e] = a.q_scale * (a.q_weight ? __ldg(a.q_weight + e) : 1.f);
                    weight_s[1][e] = a.k_weight ? __ldg(a.k_weight + e) : 1.f;
                }
            }
            if (ROTATION != NO_ROTATION) {
                for (int j = threadIdx.x; j < tokens * half; j += THREADS) {
                    const int t = j / half, f = j - t * half;
                    const double turns = (double)__ldg(a.positions + token0 + t) * (double)__ldg(a.inv_freq + f) * 0.15915494309189533577;
                    float s, c;
                    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
                    float* to = turn_s + 3 * t * half + f;
                    to[0] = c;
                    to[half] = s;
                    to[2 * half] = -s;
                }
            }
            if (weights || ROTATION != NO_ROTATION) __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = base + i * GROUPS + group, tok = token_of(row), head = row - tok * a.heads;
            const bool is_q = head < a.hq;
            float2 x[CHUNKS][4];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) raw[i][c].unpack(x[c]);
            float scale = is_q && !weights ? a.q_scale : 1.f;
            if (a.norm != ONELA_NORM_NONE) {
                float2 sums = make_float2(0.f, 0.f);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums = __ffma2_rn(x[c][e], x[c][e], sums);
                float sum = sums.x + sums.y;
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                scale *= rsqrtf(fmaf(sum, a.sum_weight, a.eps));
            }
            if (weights) {
                const float* w = weight_s[is_q ? 0 : 1] + at;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {        // (what lies behind the row's end is not stored)
                        const float4 w4 = *reinterpret_cast<const float4*>(w + c * (LPR * 8) + 2 * e);
                        x[c][e] = __fmul2_rn(x[c][e], __fmul2_rn(make_float2(w4.x, w4.y), make_float2(scale, scale)));
                        x[c][e + 1] = __fmul2_rn(x[c][e + 1], __fmul2_rn(make_float2(w4.z, w4.w), make_float2(scale, scale)));
                    }
            } else {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[c][e] = __fmul2_rn(x[c][e], make_float2(scale, scale));
            }
            if (ROTATION != NO_ROTATION) {
                const float* cs = turn_s + 3 * (tok < tokens ? tok : 0) * half;
                if (ROTATION == INTERLEAVED) {
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
                        const int el = at + c * (LPR * 8);
                        if (el < a.rotary) {
                            const float4 co = *reinterpret_cast<const float4*>(cs + el / 2), si = *reinterpret_cast<const float4*>(cs + half + el / 2);
                            const float cv[4] = {co.x, co.y, co.z, co.w}, sv[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[c][e] = make_float2(x[c][e].x * cv[e] - x[c][e].y * sv[e], x[c][e].y * cv[e] + x[c][e].x * sv[e]);
                        }
                    }
                } else {
                    // x (of the lower or upper half) with its partner y
                    auto turn = [&](float2* v, const float2* y, int f, bool low) {
                        const float *cp = cs + f, *sp = cp + (low ? 2 * half : half);
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const float4 co = *reinterpret_cast<const float4*>(cp + 2 * e), si = *reinterpret_cast<const float4*>(sp + 2 * e);
                            v[e] = __ffma2_rn(v[e], make_float2(co.x, co.y), __fmul2_rn(y[e], make_float2(si.x, si.y)));
                            v[e + 1] = __ffma2_rn(v[e + 1], make_float2(co.z, co.w), __fmul2_rn(y[e + 1], make_float2(si.z, si.w)));
                        }
                    };
                    if (CHUNKS == 2 && half == LPR * 8) {   // the halves are a lane's two pieces
                        float2 lower[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) lower[e] = x[0][e];
                        turn(x[0], x[CHUNKS - 1], at, true);
                        turn(x[CHUNKS - 1], lower, at, false);
                    } else {                                // both halves lie in the lanes' first pieces
                        const bool low = at < half, turned = at < a.rotary;
                        const int other = !turned ? lane : low ? lane + half / 8 : lane - half / 8;
                        float2 y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            y[e].x = __shfl_sync(0xffffffffu, x[0][e].x, other, LPR);
                            y[e].y = __shfl_sync(0xffffffffu, x[0][e].y, other, LPR);
                        }
                        if (turned) turn(x[0], y, low ? at : at - half, low);
                    }
                }
            }
            T* p = (is_q ? q_out : k_out) + (tok * (is_q ? q_out_step : k_out_step) + (is_q ? head : head - a.hq) * a.dim);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (row < rows && at + c * (LPR * 8) < a.dim) {
                    const float y[8] = {x[c][0].x, x[c][0].y, x[c][1].x, x[c][1].y, x[c][2].x, x[c][2].y, x[c][3].x, x[c][3].y};
                    store_out<T, 8>(p + c * (LPR * 8), y);
                }
            }
        }
    }
}

template <typename T, int LPR, int CHUNKS>
cudaError_t launch_shape(NormArgs a, cudaStream_t stream) {
    // tokens per CTA: the fewest passes of rows in a row on one place of an SM (whole waves of CTAs while there are few)
    constexpr int TILE = THREADS / LPR * (ROWS_IN_FLIGHT / CHUNKS), MOST = 16, PLACES = 148 * OCCUPANCY;
    a.tokens = 1;
    double best = 1e30;
    for (int t = 1; t <= MOST; ++t) {
        // (a token's number within the CTA is a product: rows below 2^16; offsets within the CTA have 32 bits)
        if (t > 1 && ((long long)t * a.heads + TILE > 65535 || a.heads == 1 || std::max(std::max(a.q_stride, a.k_stride), std::max(a.q_out_stride, a.k_out_stride)) > (1ll << 26))) break;
        const long long passes = ((long long)t * a.heads + TILE - 1) / TILE;
        const double waves = (double)((a.n_tokens + t - 1) / t) / PLACES, cost = (double)passes * (waves < 4 ? std::ceil(waves) : waves);
        if (cost < best * (1 - 1e-9)) {
            best = cost;
            a.tokens = t;
        }
    }
    a.magic = a.tokens > 1 ? (uint32_t)(((1ull << 32) + a.heads - 1) / a.heads) : 0;      // row * magic / 2^32 = row / heads; one token: 0
    const dim3 grid((unsigned)((a.n_tokens + a.tokens - 1) / a.tokens));
    const size_t smem = (size_t)a.tokens * a.rotary / 2 * 3 * sizeof(float);
    return a.rotary == 0     ? launch_dependent(norm_rotate_kernel<T, LPR, CHUNKS, NO_ROTATION>, grid, dim3(THREADS), smem, stream, a)
           : !a.interleaved ? launch_dependent(norm_rotate_kernel<T, LPR, CHUNKS, HALVES>, grid, dim3(THREADS), smem, stream, a)
                            : launch_dependent(norm_rotate_kernel<T, LPR, CHUNKS, INTERLEAVED>, grid, dim3(THREADS), smem, stream, a);
}
// Two pieces per lane where a rotation's partners then share a lane or lie in the first pieces: half the lanes' work per row that
// does not depend on its width.
template <typename T>
cudaError_t launch_t(const NormArgs& a, cudaStream_t stream) {
    const int lpr = a.dim <= 64 ? 4 : a.dim <= 128 ? 8 : 16;
    const bool two = a.dim > 32 && (a.rotary == 0 || a.interleaved || a.rotary <= lpr * 8 || a.rotary == lpr * 16);
    if (a.dim <= 32) return launch_shape<T, 4, 1>(a, stream);
    if (a.dim <= 64) return two ? launch_shape<T, 4, 2>(a, stream) : launch_shape<T, 8, 1>(a, stream);
    if (a.dim <= 128) return two ? launch_shape<T, 8, 2>(a, stream) : launch_shape<T, 16, 1>(a, stream);
    return two ? launch_shape<T, 16, 2>(a, stream) : launch_shape<T, 32, 1>(a, stream);
}

}  // namespace
}  // namespace onela

extern "C" onela_status onela_norm_rotate(const onela_norm_rotate_args* g, void* stream) {
    using namespace onela;
    if (!g) return ONELA_E_INVAL;
    if (g->dtype != ONELA_DTYPE_F32 && g->dtype != ONELA_DTYPE_BF16) return ONELA_E_INVAL;
    if (g->norm != ONELA_NORM_NONE && g->norm != ONELA_NORM_L2 && g->norm != ONELA_NORM_RMS) return ONELA_E_INVAL;
    const long long es = g->dtype == ONELA_DTYPE_BF16 ? 2 : 4;
    constexpr int32_t MAX_HEADS = 1 << 20;
    if (g->n_tokens < 0 || g->num_q_heads < 0 || g->num_k_heads < 0 || g->head_dim < 1) return ONELA_E_INVAL;
    if (g->head_dim % 8 != 0 || g->head_dim > 256) return ONELA_E_UNSUPPORTED;
    if (g->rotary_dim < 0 || g->rotary_dim > g->head_dim) return ONELA_E_INVAL;
    if (g->rotary_dim % 16 != 0) return ONELA_E_UNSUPPORTED;
    if (!(g->eps >= 0.f)) return ONELA_E_INVAL;
    if (g->n_tokens == 0 || (g->num_q_heads == 0 && g->num_k_heads == 0)) return ONELA_OK;
    if (g->n_tokens > 0x7fffffffll || g->num_q_heads > MAX_HEADS || g->num_k_heads > MAX_HEADS) return ONELA_E_CAPACITY;      // CTAs of one launch, 32-bit offsets within a token
    if (g->rotary_dim > 0 && (!g->positions_dev || !g->inv_freq_dev)) return ONELA_E_INVAL;
    if (!aligned16(g->q_weight_dev) || !aligned16(g->k_weight_dev) || !aligned4(g->positions_dev, g->inv_freq_dev)) return ONELA_E_INVAL;
    const Rows set[4] = {{static_cast<const char*>(g->q_dev), g->q_stride * es, (long long)g->num_q_heads * g->head_dim * es, g->n_tokens},
                         {static_cast<const char*>(g->k_dev), g->k_stride * es, (long long)g->num_k_heads * g->head_dim * es, g->n_tokens},
                         {static_cast<const char*>(g->q_out_dev), g->q_out_stride * es, (long long)g->num_q_heads * g->head_dim * es, g->n_tokens},
                         {static_cast<const char*>(g->k_out_dev), g->k_out_stride * es, (long long)g->num_k_heads * g->head_dim * es, g->n_tokens}};
    for (const Rows& r : set) {
        if (r.extent == 0) continue;
        if (!r.base || !aligned16(r.base) || r.stride < r.extent || r.stride >= (1ll << 40) || r.stride % 16 != 0) return ONELA_E_INVAL;
    }
    for (int o = 2; o < 4; ++o)
        for (int i = 0; i < 4; ++i) {
            if (i == o || (i == o - 2 && set[i].base == set[o].base && set[i].stride == set[o].stride)) continue;      // in place
            if (share_bytes(set[i], set[o])) return ONELA_E_INVAL;
        }
    NormArgs a{g->q_dev, g->k_dev, g->q_out_dev, g->k_out_dev, nullptr, nullptr, g->positions_dev, g->inv_freq_dev, g->q_stride, g->k_stride, g->q_out_stride, g->k_out_stride,
               g->n_tokens, g->num_q_heads, g->num_q_heads + g->num_k_heads, g->head_dim, g->rotary_dim, g->interleaved != 0, g->norm, g->eps, g->q_scale, g->norm == ONELA_NORM_RMS ? 1.f / (float)g->head_dim : 1.f, 1, 0};
    if (g->norm == ONELA_NORM_RMS) {
        a.q_weight = g->q_weight_dev;
        a.k_weight = g->k_weight_dev;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = g->dtype == ONELA_DTYPE_BF16 ? launch_t<__nv_bfloat16>(a, s) : launch_t<float>(a, s);
    return e == cudaSuccess ? ONELA_OK : ONELA_E_CUDA;
}
