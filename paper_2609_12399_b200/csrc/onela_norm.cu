// Norms of queries and keys for each head with the rotation by position in the same pass (onela_norm_rotate).
//
// A head vector x of d elements becomes y = x / sqrt(sum x^2 + eps) or x / sqrt(mean x^2 + eps) * w, its first r elements turn in pairs
// by the angle position * inv_freq[i], queries are scaled.  Every element is read once and written once, so HBM bounds it.
//
// A row is one (token, head), queries' and keys' heads of a token behind one another; 4 to 32 lanes share it, 8 elements (16 bytes of
// bf16, 32 of fp32) each, and a thread has ROWS rows in flight.  The angles belong to the token: a CTA, whose rows are consecutive, forms
// cosine and sine of its few tokens once in shared memory.  position * inv_freq is exact in 64 bits (31 + 24 bits; two more than fit are
// rounded), reduced there to a fraction of a turn, and only the fraction goes through the fp32 functions, so far positions lose nothing.
// Elements i and i + r / 2 lie in different lanes of a row (r is a multiple of 16), 8 shuffles away.
#include <algorithm>

#include "onela_internal.h"
#include "onela_layout.cuh"

namespace onela {
namespace {

constexpr int THREADS = 256, ROWS = 4;

struct NormArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const float *q_weight, *k_weight;
    const int32_t* positions;
    const float* inv_freq;
    long long q_stride, k_stride, q_out_stride, k_out_stride, n_tokens;
    int32_t hq, heads, dim, rotary, interleaved, norm;
    float eps, q_scale;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* x) {
    Vec16<float>::load(p, x);
    Vec16<float>::load(p + 4, x + 4);
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float* x) { Vec16<__nv_bfloat16>::load(p, x); }

template <typename T, int LPR>
__global__ void __launch_bounds__(THREADS) norm_rotate_kernel(const NormArgs a) {
    constexpr int GROUPS = THREADS / LPR, TILE = GROUPS * ROWS;
    extern __shared__ float turn_s[];                       // [tokens of the CTA][cos r / 2 | sin r / 2]
    const int half = a.rotary / 2;
    const long long first = (long long)blockIdx.x * TILE, token0 = first / a.heads;
    const int head0 = (int)(first - token0 * a.heads);
    const long long left = a.n_tokens - token0;             // tokens from the CTA's first one on
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR, at = lane * 8;
    const bool inside = at < a.dim;
    float x[ROWS][8];
    int tok[ROWS], head[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int row = head0 + i * GROUPS + group;
        tok[i] = row / a.heads;
        head[i] = row - tok[i] * a.heads;
        if (tok[i] >= left) tok[i] = -1;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
        if (tok[i] >= 0 && inside) {
            const bool is_q = head[i] < a.hq;
            const T* p = is_q ? static_cast<const T*>(a.q) + (token0 + tok[i]) * a.q_stride + (long long)head[i] * a.dim
                              : static_cast<const T*>(a.k) + (token0 + tok[i]) * a.k_stride + (long long)(head[i] - a.hq) * a.dim;
            load8(p + at, x[i]);
        }
    }
    if (half > 0) {
        const int span = (int)min(left, (long long)((head0 + TILE - 1) / a.heads + 1));
        for (int j = threadIdx.x; j < span * half; j += THREADS) {
            const int t = j / half, f = j - t * half;
            const double turns = (double)a.positions[token0 + t] * (double)a.inv_freq[f] * 0.15915494309189533577;
            float s, c;
            sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
            turn_s[2 * t * half + f] = c;
            turn_s[(2 * t + 1) * half + f] = s;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const bool is_q = head[i] < a.hq;
        if (a.norm != ONELA_NORM_NONE) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[i][e], x[i][e], sum);
#pragma unroll
            for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float n = 1.f / sqrtf(a.norm == ONELA_NORM_L2 ? sum + a.eps : sum / (float)a.dim + a.eps);
            const float* w = is_q ? a.q_weight : a.k_weight;
            if (w && inside) {
                float wx[8];
                load8(w + at, wx);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= n * wx[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= n;
            }
        }
        if (half > 0) {
            const float *cs = turn_s + 2 * max(tok[i], 0) * half, *sn = cs + half;
            if (a.interleaved) {
                if (at < a.rotary) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float c = cs[(at + e) >> 1], s = sn[(at + e) >> 1], u = x[i][e], v = x[i][e + 1];
                        x[i][e] = u * c - v * s;
                        x[i][e + 1] = v * c + u * s;
                    }
                }
            } else {
                const bool low = at < half, turned = at < a.rotary;
                const int other = low ? lane + half / 8 : lane - half / 8;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __shfl_sync(0xffffffffu, x[i][e], turned ? other : lane, LPR);
                if (turned) {
                    const int f = low ? at : at - half;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float c = cs[f + e], s = low ? -sn[f + e] : sn[f + e];
                        x[i][e] = x[i][e] * c + y[e] * s;
                    }
                }
            }
        }
        if (tok[i] >= 0 && inside) {
            if (is_q) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= a.q_scale;
            }
            T* p = is_q ? static_cast<T*>(a.q_out) + (token0 + tok[i]) * a.q_out_stride + (long long)head[i] * a.dim
                        : static_cast<T*>(a.k_out) + (token0 + tok[i]) * a.k_out_stride + (long long)(head[i] - a.hq) * a.dim;
            store_out<T, 8>(p + at, x[i]);
        }
    }
}

template <typename T, int LPR>
cudaError_t launch_lpr(const NormArgs& a, cudaStream_t stream) {
    constexpr int TILE = THREADS / LPR * ROWS;
    const long long rows = a.n_tokens * a.heads, ctas = (rows + TILE - 1) / TILE;
    const size_t smem = (size_t)a.rotary * sizeof(float) * std::min<long long>(a.n_tokens, (a.heads - 1 + TILE - 1) / a.heads + 1);
    static_assert(THREADS / 4 * ROWS * 32 * 4 <= 48 * 1024, "one head of the narrowest row: cosines and sines of a CTA");
    return launch_dependent(norm_rotate_kernel<T, LPR>, dim3((unsigned)ctas), dim3(THREADS), smem, stream, a);
}
template <typename T>
cudaError_t launch_t(const NormArgs& a, cudaStream_t stream) {
    if (a.dim <= 32) return launch_lpr<T, 4>(a, stream);
    if (a.dim <= 64) return launch_lpr<T, 8>(a, stream);
    if (a.dim <= 128) return launch_lpr<T, 16>(a, stream);
    return launch_lpr<T, 32>(a, stream);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Rows [base + i stride, + extent) in bytes, i < n
struct Rows {
    const char* base;
    long long stride, extent, n;
    long long span() const { return (n - 1) * stride + extent; }
};
// Whether two sets of rows share a byte (sets of different strides: whether their spans do).
bool share_bytes(const Rows& x, const Rows& y) {
    if (x.extent == 0 || y.extent == 0) return false;
    const Rows &a = x.base <= y.base ? x : y, &b = x.base <= y.base ? y : x;
    const long long off = b.base - a.base;
    if (off >= a.span()) return false;
    if (a.stride != b.stride) return true;
    const long long within = off % a.stride;         // b's first row in a's row of the same number, or of a later one
    if (within < a.extent && off / a.stride < a.n) return true;
    return within + b.extent > a.stride && off / a.stride + 1 < a.n;
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
    if (g->n_tokens < 0 || g->num_q_heads < 0 || g->num_k_heads < 0 || g->num_q_heads > MAX_HEADS || g->num_k_heads > MAX_HEADS || g->head_dim < 1) return ONELA_E_INVAL;
    if (g->head_dim % 8 != 0 || g->head_dim > 256) return ONELA_E_UNSUPPORTED;
    if (g->rotary_dim < 0 || g->rotary_dim > g->head_dim) return ONELA_E_INVAL;
    if (g->rotary_dim % 16 != 0) return ONELA_E_UNSUPPORTED;
    if (!(g->eps >= 0.f)) return ONELA_E_INVAL;
    if (g->n_tokens == 0 || g->num_q_heads + g->num_k_heads == 0) return ONELA_OK;
    const long long heads = (long long)g->num_q_heads + g->num_k_heads;
    if (g->n_tokens > (1ll << 40) / heads || g->n_tokens * heads / (THREADS / 32 * ROWS) >= 0x7fffffffll) return ONELA_E_CAPACITY;    // CTAs of one launch
    if (g->rotary_dim > 0 && (!g->positions_dev || !g->inv_freq_dev)) return ONELA_E_INVAL;
    if (!aligned16(g->q_weight_dev) || !aligned16(g->k_weight_dev)) return ONELA_E_INVAL;
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
               g->n_tokens, g->num_q_heads, g->num_q_heads + g->num_k_heads, g->head_dim, g->rotary_dim, g->interleaved != 0, g->norm, g->eps, g->q_scale};
    if (g->norm == ONELA_NORM_RMS) {
        a.q_weight = g->q_weight_dev;
        a.k_weight = g->k_weight_dev;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = g->dtype == ONELA_DTYPE_BF16 ? launch_t<__nv_bfloat16>(a, s) : launch_t<float>(a, s);
    return e == cudaSuccess ? ONELA_OK : ONELA_E_CUDA;
}
