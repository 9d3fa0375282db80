// Device helpers of the kernels that work on chunks of 64 tokens (onela_prefill.cu, onela_delta_chunk.cu): operand layouts, fp16
// operands in parts, small triangular products in shared memory.
#pragma once

#include "onela_sm100.cuh"

namespace onela {
namespace chunk {

using sm100::pack_f16x2;
using sm100::smem_u32;
using sm100::tmem_st16;

constexpr int C = 64;              // tokens per chunk
constexpr int TILE = C * 128;      // bytes of one K-major operand block: 64 rows of 64 fp16
constexpr int AP = C + 4;          // pitch (floats) of the C x C matrix: 16-byte rows

// MN-major operand, 128-byte swizzle: rows (K index) of 64 elements, 8-row groups 1024 bytes apart, blocks of 64
// elements along M or N `block` bytes apart.
__device__ __forceinline__ uint64_t umma_desc_mn(uint32_t smem_addr, uint32_t block) {
    return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}
constexpr uint32_t A_MN_MAJOR = 1u << 15, B_MN_MAJOR = 1u << 16;     // instruction descriptor: operand is MN-major
constexpr uint32_t BF16_OPERANDS = (1u << 7) | (1u << 10);           // ... both are bf16

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// Two numbers times a power of two as fp16 numbers hi + lo (+ low), packed.  (Rounding hi to a fixed grid instead would make
// sums of hi x hi products exact, but leaves every lo as large as the row's largest element allows.)
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16x2(a, b);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    lo = pack_f16x2(a - h.x, b - h.y);
}
__device__ __forceinline__ void split3(float a, float b, uint32_t& hi, uint32_t& lo, uint32_t& low) {
    hi = pack_f16x2(a, b);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    const float ra = a - h.x, rb = b - h.y;
    lo = pack_f16x2(ra, rb);
    const float2 l = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    low = pack_f16x2(ra - l.x, rb - l.y);
}
// Sixteen numbers times `scale` in two parts or (low not null) three; `keep`: what the low part gives on top (see KEEP_DELTA).
__device__ __forceinline__ void split16(const float* x, float scale, uint32_t* hi, uint32_t* lo, float keep = 0.f, uint32_t* low = nullptr) {
    const float2 sc = make_float2(scale, scale), kp = make_float2(keep, keep);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 y = __fmul2_rn(make_float2(x[2 * e], x[2 * e + 1]), sc);
        hi[e] = pack_f16x2(y.x, y.y);
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi[e]));
        float2 l = __fadd2_rn(y, make_float2(-h.x, -h.y));
        if (keep != 0.f) l = __ffma2_rn(y, kp, l);
        lo[e] = pack_f16x2(l.x, l.y);
        if (low) {
            const float2 q = __half22float2(*reinterpret_cast<const __half2*>(&lo[e]));
            const float2 r = __fadd2_rn(l, make_float2(-q.x, -q.y));
            low[e] = pack_f16x2(r.x, r.y);
        }
    }
}
// Two fp32 numbers as the sum of three bf16 ones each, packed: eight bits at a time, exact.  (The first is cut off, so that the
// largest numbers stay finite, the second rounded, so that the third has either sign and products left out have no bias.)
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t (&part)[3]) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    part[0] = __byte_perm(ua, ub, 0x7632);
    const float ra = a - __uint_as_float(ua & 0xffff0000u), rb = b - __uint_as_float(ub & 0xffff0000u);
    part[1] = sm100::pack_bf16x2(ra, rb);
    float ma, mb;
    unpack_bf16x2(part[1], ma, mb);
    part[2] = sm100::pack_bf16x2(ra - ma, rb - mb);
}
// ... as one K step of a tensor-memory A operand: columns [0, 8) hi, [8, 16) lo
__device__ __forceinline__ void split_to_tmem(uint32_t taddr, const float* x, float scale) {
    uint32_t w[16];
    split16(x, scale, w, w + 8);
    tmem_st16(taddr, w);
}
// ... of numbers that are in range as they are
__device__ __forceinline__ void split_to_tmem(uint32_t taddr, const float* x) {
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = pack_f16x2(x[2 * e], x[2 * e + 1]);
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[e])), l = __fadd2_rn(make_float2(x[2 * e], x[2 * e + 1]), make_float2(-h.x, -h.y));
        w[8 + e] = pack_f16x2(l.x, l.y);
    }
    tmem_st16(taddr, w);
}

// acc[r] = sum over l < N of rows[r][l] cols[l]: eight rows (pitch AP, read as broadcast vectors) times this lane's column, the
// even and the odd l in the two halves of packed multiply-adds.  UNROLL steps of four l at a time: all of them at dk <= 64 (5000
// tokens x 16 heads of 32 x 32 fp32 83.2 -> 79.5 us, 6000 x 32 heads of 64 x 64 bf16 124.0 -> 119.5, although that one then spills 12
// bytes: four steps, which do not, 1 - 2 % slower from 1021 to 16 384 tokens), two at dk = 128, whose roles miss the instruction cache
// (16 384 tokens 434.7 -> 429.5; four 439.6, eight 454.2).  Error against 64
// bits: 0.3 % smaller on the mean of fourteen shapes, none more than 0.5 % larger.
template <int N, int UNROLL>
__device__ __forceinline__ void rows8(float* acc, const float* rows, const float* cols, int pitch) {
    float2 sum[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) sum[r] = make_float2(0.f, 0.f);
#pragma unroll UNROLL
    for (int l = 0; l < N; l += 4) {
        const float2 t0 = make_float2(cols[l * pitch], cols[(l + 1) * pitch]), t1 = make_float2(cols[(l + 2) * pitch], cols[(l + 3) * pitch]);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const float4 q = *reinterpret_cast<const float4*>(rows + r * AP + l);
            sum[r] = __ffma2_rn(make_float2(q.x, q.y), t0, __ffma2_rn(make_float2(q.z, q.w), t1, sum[r]));
        }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) acc[r] = sum[r].x + sum[r].y;
}

}  // namespace chunk
}  // namespace onela
