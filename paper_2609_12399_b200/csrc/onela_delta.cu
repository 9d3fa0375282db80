// The gated delta rule over ragged sequences: the entry point, and the kernel that steps token by token (onela_delta_rule).
//
//      S <- a S + d k^T ,  d = b (v - a S k) ,  o = S q        per (sequence, value head)
//
// The rows of S (one per element of v) are independent, so a CTA holds a block of rows in registers: dk / 16 lanes share a row,
// 16 elements each.  Per token and row two dot products with the OLD row, S k and S q (their reductions run side by side), then
// d, o = a (S q) + d (k . q) and the row's update; all in fp32.  One token: the state's bytes, read once and written once, bound it.
// Many tokens: the chain of a token's latencies (the next token's inputs are on their way meanwhile), so long sequences go to the
// chunked kernel (onela_delta_chunk.cu).
//
// Measured: 64 sequences x 32 heads of 128 x 128, one token, 43.5 us (5.9 TB/s, 0.92 of the measured copy); 16 heads of one sequence 3.7 us, a launch;
// 37 sequences x 16 heads of 64 x 64 fp32, five tokens, 9.5 us.
//
// A lane group works on PASSES rows.  Four, so that a warp has 4 x 512 bytes x 4 of state in flight, where the call fills the GPU; one,
// four times the CTAs, where it does not.
#include <algorithm>

#include "onela_delta.cuh"
#include "onela_layout.cuh"

namespace onela {
namespace {

constexpr int WARPS = 4;
// Tokens of the longest sequence from which the chunked kernel is the faster one.  Measured, us token by token / in chunks, 16 heads, one sequence, four, 37:
// 128 x 128 bf16, 24 tokens 11.3 / 18.7, 17.3 / 19.1, 72 / 76; 32: 14.5 / 18.8, 22.2 / 19.2, 93 / 77; 48: 20.5 / 19.1, 31.6 / 19.5, 135 / 78 (32 heads, four of 16:
// 20.2 / 19.5); 128 x 128 fp32, 32 tokens 11.0 / 19.1, 19.0 / 19.4, 88 / 79; 64 x 64 bf16, 24 tokens 10.6 / 12.7, 11.1 / 13.0, 42 / 53; 32: 13.6 / 12.8, 14.1 / 13.1, 54 / 53.
// Narrow heads in fp32 take fewer instructions token by token and more in chunks: 64 x 64, 40 tokens 12.9 / 13.7, 13.5 / 14.0, 48 / 56; 48: 15.2 / 13.7, 15.7 / 14.0, 57 / 56;
// 32 x 32, 40 tokens 12.4 / 11.4, 12.8 / 11.8, 45 / 47.
inline long long chunked_from(int32_t dtype, int32_t dk) { return dtype == ONELA_DTYPE_F32 && dk <= 64 ? 44 : 32; }

template <typename T>
__device__ __forceinline__ void load4(const T* p, float* x);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float* x) { Vec16<float>::load(p, x); }
template <>
__device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, float* x) {
    const uint2 w = __ldg(reinterpret_cast<const uint2*>(p));
    unpack_bf16x2(w.x, x[0], x[1]);
    unpack_bf16x2(w.y, x[2], x[3]);
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, float* p) { *p = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

// What a lane needs of a token: its 16 elements of k and q, its rows' values, the gates.
template <typename T, int LPR, int PASSES>
struct Token {
    float k[16], q[16], v[PASSES], alpha, beta;
    __device__ __forceinline__ void load(const DeltaArgs& a, long long t, int hk, int hv, int lane, int row0, int row_step) {
        const T *kp = static_cast<const T*>(a.k) + t * a.k_stride + (long long)hk * (LPR * 16) + lane * 4;
        const T *qp = static_cast<const T*>(a.q) + t * a.q_stride + (long long)hk * (LPR * 16) + lane * 4;
        const T* vp = static_cast<const T*>(a.v) + t * a.v_stride + (long long)hv * a.dv;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            load4(kp + c * (LPR * 4), k + 4 * c);
            load4(qp + c * (LPR * 4), q + 4 * c);
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int row = row0 + p * row_step;
            v[p] = row < a.dv ? to_float(__ldg(vp + row)) : 0.f;
        }
        alpha = __ldg(a.alpha + t * a.gate_stride + hv);
        beta = __ldg(a.beta + t * a.gate_stride + hv);
    }
};

template <int LPR>
__device__ __forceinline__ float sum_of_lanes(float x) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <int DK, typename T, int PASSES>
__global__ void __launch_bounds__(WARPS * 32) delta_step_kernel(const DeltaArgs a) {
    constexpr int LPR = DK / 16, STEP = 32 / LPR, ROWS = STEP * PASSES;      // lanes per row, rows per pass and per warp
    const int warp = threadIdx.x / 32, lane = threadIdx.x % LPR, group = threadIdx.x % 32 / LPR;
    const int i = blockIdx.z, hv = blockIdx.y, hk = hv / (a.Hv / a.Hk);
    const int row0 = (blockIdx.x * WARPS + warp) * ROWS + group;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Sequence s = read_sequence(a, i, blockIdx.x == 0 && hv == 0);
    if (!s.live) return;                                                     // (the whole CTA)
    float S[PASSES][16];
    float* state = a.states + s.slot * a.state_stride + (long long)hv * a.dv * DK + lane * 4;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * STEP;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < a.dv && !s.fresh) x = __ldcs(reinterpret_cast<const float4*>(state + (long long)row * DK + c * (LPR * 4)));
            S[p][4 * c] = x.x; S[p][4 * c + 1] = x.y; S[p][4 * c + 2] = x.z; S[p][4 * c + 3] = x.w;
        }
    }
    Token<T, LPR, PASSES> next;
    if (s.length > 0) next.load(a, s.begin, hk, hv, lane, row0, STEP);
    if (__syncthreads_or(taken_before(a, i, s, threadIdx.x, WARPS * 32))) {
        if (blockIdx.x == 0 && hv == 0 && threadIdx.x == 0) report_taken(a, i);
        return;
    }
    for (int t = 0; t < s.length; ++t) {
        const Token<T, LPR, PASSES> now = next;
        if (t + 1 < s.length) next.load(a, s.begin + t + 1, hk, hv, lane, row0, STEP);
        float sk[PASSES], sq[PASSES], kq = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) kq = fmaf(now.k[e], now.q[e], kq);
        kq = sum_of_lanes<LPR>(kq);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            float2 dk = make_float2(0.f, 0.f), dq = make_float2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float2 x = make_float2(S[p][e], S[p][e + 1]);
                dk = __ffma2_rn(x, make_float2(now.k[e], now.k[e + 1]), dk);
                dq = __ffma2_rn(x, make_float2(now.q[e], now.q[e + 1]), dq);
            }
            sk[p] = dk.x + dk.y;
            sq[p] = dq.x + dq.y;
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            sk[p] = sum_of_lanes<LPR>(sk[p]);
            sq[p] = sum_of_lanes<LPR>(sq[p]);
        }
        T* out = static_cast<T*>(a.out) + (s.begin + t) * a.out_stride + (long long)hv * a.dv;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const float d = now.beta * (now.v[p] - now.alpha * sk[p]);
            const float2 d2 = make_float2(d, d), al = make_float2(now.alpha, now.alpha);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float2 x = __ffma2_rn(d2, make_float2(now.k[e], now.k[e + 1]), __fmul2_rn(al, make_float2(S[p][e], S[p][e + 1])));
                S[p][e] = x.x;
                S[p][e + 1] = x.y;
            }
            const int row = row0 + p * STEP;
            if (lane == 0 && row < a.dv) from_float(fmaf(d, kq, now.alpha * sq[p]), out + row);
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * STEP;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (row < a.dv) __stcs(reinterpret_cast<float4*>(state + (long long)row * DK + c * (LPR * 4)), make_float4(S[p][4 * c], S[p][4 * c + 1], S[p][4 * c + 2], S[p][4 * c + 3]));
    }
}

template <int DK, typename T, int PASSES>
cudaError_t launch_passes(const DeltaArgs& a, cudaStream_t stream) {
    constexpr int ROWS = WARPS * PASSES * (32 / (DK / 16));
    const dim3 grid((a.dv + ROWS - 1) / ROWS, a.Hv, a.num_sequences);
    return launch_dependent(delta_step_kernel<DK, T, PASSES>, grid, dim3(WARPS * 32), 0, stream, a);
}
template <int DK, typename T>
cudaError_t launch_step(const DeltaArgs& a, cudaStream_t stream) {
    constexpr int ROWS = WARPS * 4 * (32 / (DK / 16));
    const long long ctas = (long long)((a.dv + ROWS - 1) / ROWS) * a.Hv * a.num_sequences;
    return ctas >= 256 ? launch_passes<DK, T, 4>(a, stream) : launch_passes<DK, T, 1>(a, stream);
}
template <typename T>
cudaError_t launch_step_t(const DeltaArgs& a, cudaStream_t stream) {
    switch (a.dk) {
        case 32: return launch_step<32, T>(a, stream);
        case 64: return launch_step<64, T>(a, stream);
        case 128: return launch_step<128, T>(a, stream);
        default: return launch_step<256, T>(a, stream);
    }
}

}  // namespace
}  // namespace onela

extern "C" onela_status onela_delta_rule(const onela_delta_rule_args* g, void* stream) {
    using namespace onela;
    if (!g) return ONELA_E_INVAL;
    if (g->dtype != ONELA_DTYPE_F32 && g->dtype != ONELA_DTYPE_BF16) return ONELA_E_INVAL;
    if (g->n_tokens < 0 || g->num_sequences < 0 || g->num_states < 0 || g->max_tokens < 0 || g->num_heads < 1 || g->num_v_heads < 1) return ONELA_E_INVAL;
    if (g->num_v_heads % g->num_heads != 0) return ONELA_E_INVAL;
    if (g->dk != 32 && g->dk != 64 && g->dk != 128 && g->dk != 256) return ONELA_E_UNSUPPORTED;
    if (g->dv < 32 || g->dv % 32 != 0 || g->dv > 512) return ONELA_E_UNSUPPORTED;
    if (g->num_sequences > 65535 || g->num_v_heads > 65535 || g->n_tokens > 0x7fffff00ll) return ONELA_E_CAPACITY;
    if (!g->starts_dev && g->n_tokens != g->num_sequences) return ONELA_E_INVAL;
    if (!g->slots_dev && g->num_states < g->num_sequences) return ONELA_E_INVAL;
    if (!aligned4(g->alpha_dev, g->beta_dev, g->starts_dev, g->slots_dev, g->fresh_dev, g->status_dev)) return ONELA_E_INVAL;
    if (g->num_sequences == 0) return ONELA_OK;
    const long long es = g->dtype == ONELA_DTYPE_BF16 ? 2 : 4, big = 1ll << 40;
    auto rows = [](const void* p, long long stride, long long extent, long long size, long long n) {
        return Rows{static_cast<const char*>(p), stride * size, extent * size, n};
    };
    // inputs, outputs, states
    const Rows set[5] = {rows(g->q_dev, g->q_stride, (long long)g->num_heads * g->dk, es, g->n_tokens), rows(g->k_dev, g->k_stride, (long long)g->num_heads * g->dk, es, g->n_tokens),
                         rows(g->v_dev, g->v_stride, (long long)g->num_v_heads * g->dv, es, g->n_tokens), rows(g->out_dev, g->out_stride, (long long)g->num_v_heads * g->dv, es, g->n_tokens),
                         rows(g->states_dev, g->state_stride, (long long)g->num_v_heads * g->dv * g->dk, 4, g->num_states)};
    for (const Rows& r : set)
        if (r.n > 0 && (!r.base || !aligned16(r.base) || r.stride < r.extent || r.stride >= big || r.stride % 16 != 0)) return ONELA_E_INVAL;
    if (g->n_tokens > 0 && (!g->alpha_dev || !g->beta_dev || g->gate_stride < g->num_v_heads || g->gate_stride >= big)) return ONELA_E_INVAL;
    for (int i = 0; i < 4; ++i)
        if ((i < 3 && share_bytes(set[i], set[3])) || share_bytes(set[i], set[4])) return ONELA_E_INVAL;
    const DeltaArgs a{g->q_dev, g->k_dev, g->v_dev, g->alpha_dev, g->beta_dev, g->states_dev, g->out_dev, g->starts_dev, g->slots_dev, g->fresh_dev, g->status_dev,
                      g->q_stride, g->k_stride, g->v_stride, g->out_stride, g->gate_stride, g->state_stride, g->n_tokens,
                      g->num_sequences, g->num_states, g->num_heads, g->num_v_heads, g->dv, g->dk, 1};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long longest = !g->starts_dev ? 1 : g->max_tokens > 0 ? g->max_tokens : g->n_tokens;
    const cudaError_t e = longest >= chunked_from(g->dtype, g->dk) && delta_chunk_supported(g->dk, g->dv) ? launch_delta_chunk(a, g->dtype, longest, s)
                          : g->dtype == ONELA_DTYPE_BF16 ? launch_step_t<__nv_bfloat16>(a, s) : launch_step_t<float>(a, s);
    return e == cudaSuccess ? ONELA_OK : ONELA_E_CUDA;
}
