// The gated delta rule over long sequences, in chunks of C = 64 tokens on the tensor cores (sm_100a): outputs of every token and the
// state behind the last (onela_delta_rule; token by token: onela_delta.cu).  dk in {32, 64, 128}, any dv.
//
// With g_i = prod_{l <= i} alpha_l inside the chunk, A_ij = beta_i (g_i / g_j)(k_i . k_j) for j < i and T = (I + A)^-1 (unit lower
// triangular; ratios are running products, nothing is divided), Eq. 1 over the chunk is (WY form of a product of Householder-like
// factors, Bischof and Van Loan 1987; with gates, Gated DeltaNet, Yang et al. 2024)
//      Z = S K^T ,  X = (V^T - Z diag(g)) diag(beta) ,  D = X T^T                         (dv x C: column i is delta_i)
//      O = S Q^T diag(g) + D P^T ,  P_ij = (g_i / g_j)(q_i . k_j) for j <= i              (dv x C)
//      S <- g_C S + D diag(g_C / g) K .
// T is applied to X, inside the chain, and not to K and V ahead of it: that costs the chain a product of 128 x 64 x 64, and
// spares the preparation two products of that size with their operands and read-backs (in onela_prefill.cu the preparation is what
// binds), and the memory of their tiles, where the queries find room.
//
// One CTA = (128 rows of the state, value head, sequence), all chunks of the sequence in order.  The state's rows lie in registers, a row in
// two threads (a half each; dk = 64: four), one in each CHAIN warpgroup; all products have the rows as M = 128 lanes:
//      S [K; Q]^T       one MMA set for Z and S Q^T (N = 128)
//      X T^T, D K, D P^T
// PREPARING warpgroups take the chunks in turn: keys and queries to an operand tile (128 rows: 64 of K, 64 of Q), [K; Q] K^T in one MMA set,
// A's and P's rows from it, T by blocks of 16 and joins, T and P as operand tiles.  An OUTPUT warpgroup brings the values into
// shared memory and forms and stores O from the two accumulators, beside the chain's next steps.  All of it is coupled by mbarriers over rings.
//
// Few long sequences leave most SMs idle, so they are cut into segments (launch_delta_chunk).  The map of a segment is affine, S -> S M + B, and M obeys the
// recurrence of S from the identity, without values.  Three launches: MAPS, every segment but the last, from zero (B; the first segment from its own
// state) and, but for the first, from the identity (M), no outputs; FOLD, the segments' states in order (delta_fold_kernel); OUTPUTS, every
// segment from its state.  The state before a segment, its predecessor's B before that, and M lie meanwhile in the segment's own rows of the caller's `out`, which OUTPUTS overwrites when it
// has read them: a segment holds enough tokens for that, or its sequence is not cut.
//
// Precision.  S, X, D and the results are fp32.  Where a product runs over the state's columns (S [K; Q]^T, [K; Q] K^T) or into them (D K) an operand's row has
// one size and its own power of two: operands are sums of two fp16 numbers (22 to 23 significant bits), keys and queries in bf16 one, exact.  (Outputs in bf16
// see all of S and D too: a query along a key that is written over, o = S k + (v - S k), cancels what is large in both.)  Along the tokens (T, P, X, D) sizes differ
// by what the gates have left, by far more than fp16's range: those operands are sums of three bf16 numbers (24 bits, fp32's range), with nothing to scale.  So
// what fades, or comes under a small key, keeps its places; only below 2^-110 they go.  (Two fp16 numbers with a scale per row instead: outputs and states wrong
// in the third digit behind 64 gates of 0.8, in the first behind 64 of 0.6.)
//
// What bounds it: a chunk takes a CTA 6.5 us (128 x 128 bf16, 16 CTAs; 7.1 with 64, 7.7 with 144, both SMs of a pair at work, which share an instruction cache; fp32 9.7, 64 x 64
// bf16 5.6, fp32 6.1).  The chain of its products and their operands is the critical path; 25 000 warp instructions, issue slots 52 % used, the tensor pipe 23 %.  4096 tokens x 16
// heads of 128 x 128 bf16: 3069 us token by token, 393 in chunks, 230 in six segments.
//   taken back or worse: D's operand for the outputs written before D K is issued (128 x 128 bf16 6.5 us -> 6.9), the six products of a triangle in a loop (+ 10 %:
//   descriptors), a barrier behind the chain's loop (the compiler lays the loop out differently: 6.5 -> 9.9); with two fp16 parts along the tokens: MMA descriptors not known to be uniform
//   (16 MMAs 5450 cycles instead of 1000), outputs stored before the accumulators are given back (period + 60 %), four chain warpgroups at dk = 128 (4096 tokens 381 -> 401),
//   values of fp32 through shared memory (T and P in one tile each: 113 -> 157)
//
// Every wait is bounded: a thread that gives up raises the abort flag and keeps meeting its team's barriers, whose OR makes the team leave
// together; ONELA_E_TIMEOUT goes to the caller's status word, if there is one, and no state is written that rests on what did not come about.  Every MMA that was issued is waited for before tensor memory is freed.
#include <algorithm>
#include <mutex>

#include "onela_chunk.cuh"
#include "onela_delta.cuh"
#include "onela_layout.cuh"
#include "onela_sm100.cuh"

namespace onela {
namespace {

using namespace chunk;
using sm100::bar_or;
using sm100::idesc_f16;
using sm100::mbar_init;
using sm100::mma_commit;
using sm100::mma_ss;
using sm100::mma_ts;
using sm100::pow2_scale;
using sm100::tmem_ld16;
using sm100::tmem_st8;
using sm100::umma_desc;

constexpr int ROWS = 128;                 // state rows per CTA
constexpr int KQ_BLOCK = 2 * TILE;        // 128 rows (64 of K, 64 of Q) of 64 fp16
constexpr int NARROW = 3, WIDE = 12;      // largest elements of fp16 operand rows: K, Q in [2^3, 2^4), S and the state's D in [2^12, 2^13)
// T and P are lower triangular, so the columns of a K step (16 tokens) are kept from their first row on: 64, 48, 32 and 16 rows, a step's two halves
// (8 columns, 16 bytes a row) one after the other; three bf16 parts.
constexpr int TRI = (64 + 48 + 32 + 16) * 32, TRI_BYTES = 3 * TRI;
__host__ __device__ constexpr int tri_at(int step) { return step * 2048 - step * (step - 1) * 256; }
constexpr int CHAIN_BARRIER = 3, OUT_BARRIER = 4;      // named barriers (1, 2: the preparing teams')

template <int D, typename T>
struct Shape {
    static constexpr bool WIDE_T = sizeof(T) == 4;
    static constexpr int KB = D > 64 ? D / 64 : 1;                 // K blocks of 64 elements
    static constexpr int PARTS = WIDE_T ? 2 : 1;                   // fp16 parts of a key, a query
    static constexpr int PREPS = WIDE_T && D == 128 ? 1 : 2;       // preparing teams
    static constexpr int K_STAGES = WIDE_T && D == 128 ? 2 : 3, T_STAGES = !WIDE_T && D == 128 ? 1 : 2, P_STAGES = 2;
    static constexpr int PREP_THREADS = 128 * PREPS, GROUPS = D == 64 ? 4 : 2, CHAIN_THREADS = 128 * GROUPS, THREADS = PREP_THREADS + CHAIN_THREADS + 128;
    static constexpr int KQ_BYTES = PARTS * KB * KQ_BLOCK;
    static constexpr bool STAGE_V = !WIDE_T;                       // values through shared memory (fp32: there is no room)
    static constexpr int V_BYTES = STAGE_V ? C * ROWS * (int)sizeof(T) : 0;
    static constexpr int O_TOKENS = 32, O_BYTES = WIDE_T ? 0 : O_TOKENS * ROWS * 2;      // outputs on their way out (bf16)
    static constexpr int A_BYTES = (C * AP * 4 + 1023) / 1024 * 1024, X_BYTES = 5 * 1024;
    // per K stage: beta g / key scale, g / query scale, beta, g_C; per P stage: weights of D's columns for the state
    static constexpr int KCO = 3 * C + 4, TCO = C;
    static constexpr int SMALL = (K_STAGES * KCO + P_STAGES * TCO + PREPS * (128 + 3 * C) + (2 * GROUPS + 2) * ROWS) * 4 + 256;
    static constexpr int SMEM = K_STAGES * KQ_BYTES + (T_STAGES + P_STAGES) * TRI_BYTES + V_BYTES + O_BYTES + PREPS * (A_BYTES + X_BYTES) + SMALL + 1024;
    static_assert(SMEM <= 232448, "shared memory");
    // tensor memory: S operand, then X operand (96), then D K | D operand for the outputs (96), in its last 64 Z before that | S Q^T (64) | D, then its operand for
    // the state (64) | D P^T (64) | [K; Q] K^T of the preparing teams (64 each; one for both where D K takes 128)
    static constexpr int X_STEP = 24;                              // columns of a K step in three bf16 parts
    static constexpr uint32_t DO_COL = D > 96 ? D : 96, Z_COL = DO_COL + 32, O1_COL = Z_COL + C, D_COL = O1_COL + C, O2_COL = D_COL + C, PREP_COL = O2_COL + C, TMEM_COLS = 512;
    static constexpr bool ONE_ACC = PREPS == 2 && D == 128;
    static_assert(PREP_COL + (ONE_ACC ? 1 : PREPS) * C <= TMEM_COLS, "tensor memory");
    // registers: 640 threads start with 96 each; at dk = 128 the chain's state rows take what the other roles leave
    static constexpr bool SPLIT_REGS = THREADS == 640 && D == 128;
    static constexpr int PREP_REGS = 72, CHAIN_REGS = 128, OUT_REGS = 80;
    static_assert(!SPLIT_REGS || 2 * PREP_REGS + 2 * CHAIN_REGS + OUT_REGS <= 5 * 96, "a split beyond the launch's registers waits for ever");
};

// the largest of m and two magnitudes, in one instruction
__device__ __forceinline__ float max3(float m, float a, float b) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ float2 pair(float x, float y) { return make_float2(x, y); }
__device__ __forceinline__ float2 pair(uint32_t x, uint32_t y) { return make_float2(__uint_as_float(x), __uint_as_float(y)); }
// (the compiler keeps what it knows to be the same in all lanes where the MMAs want it)
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// Descriptor of a K step of T or P (tri_desc of the tile plus tri_step): K-major without a swizzle, groups of eight rows 128 bytes apart, the halves as far
// as the step has rows.
__device__ __forceinline__ uint64_t tri_desc(uint32_t smem_addr) { return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46); }
__host__ __device__ constexpr uint64_t tri_step(int step) { return (uint64_t)(tri_at(step) >> 4) | ((uint64_t)(C - 16 * step) << 16); }
// Eight numbers of row `row` (fp32 bits), half `half` of K step `step`, as three bf16 parts.
__device__ __forceinline__ void store_tri(uint8_t* tile, int row, int step, int half, const uint32_t* x) {
    uint32_t part[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t w[3];
        split_bf16(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]), w);
#pragma unroll
        for (int p = 0; p < 3; ++p) part[p][e] = w[p];
    }
    uint8_t* to = tile + tri_at(step) + (half * (C - 16 * step) + row - 16 * step) * 16;
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + p * TRI) = make_uint4(part[p][0], part[p][1], part[p][2], part[p][3]);
}
// Sixteen numbers as a K step of a tensor-memory operand in three bf16 parts, eight columns each.
__device__ __forceinline__ void triple_to_tmem(uint32_t taddr, const float* x) {
    uint32_t w[24];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint32_t part[3];
        split_bf16(x[2 * e], x[2 * e + 1], part);
#pragma unroll
        for (int p = 0; p < 3; ++p) w[8 * p + e] = part[p];
    }
    tmem_st16(taddr, w);
    tmem_st8(taddr + 16, w + 16);
}

#ifdef ONELA_TEST_HOOKS
// Test-hooks build only (a second library that the product never loads): 1 + the part of a cut sequence (of sequence 0, value head 0) whose CTA of the maps'
// launch gives up when all its work is done; 0: none.
__device__ int g_hook_delta_map_fails;
#endif

enum { WHOLE, MAPS, OUTPUTS };

// The part of a sequence that a CTA works on.
struct Segment {
    int p, count;                                 // of how many
    int begin, length;                            // tokens from the sequence's first, how many
};
// Chunks that a segment must have so that its rows of `out` hold B and M, whatever the last chunk holds.
__host__ __device__ inline int least_chunks(int dk, int dv, int size) { return (int)((((long long)dv + dk) * dk * 4 + (long long)dv * size * C - 1) / ((long long)dv * size * C)) + 1; }
__device__ __forceinline__ Segment segment_of(int length, int p, int wanted, int dk, int dv, int size) {
    const int chunks = (length + C - 1) / C;
    if (wanted < 2 || chunks / wanted < least_chunks(dk, dv, size)) return {p, 1, 0, length};
    const int first = (int)((long long)chunks * p / wanted), last = (int)((long long)chunks * (p + 1) / wanted);
    return {p, wanted, first * C, min(length, last * C) - first * C};
}
// Float `at` (a multiple of 4) of what lies in the rows of `out` from `row` on, value head hv.
template <typename T>
__device__ __forceinline__ float4* scratch(const DeltaArgs& a, long long row, int hv, int at) {
    const int per = a.dv * (int)sizeof(T) / 4, r = at / per;
    return reinterpret_cast<float4*>(reinterpret_cast<float*>(static_cast<T*>(a.out) + (row + r) * a.out_stride + (long long)hv * a.dv) + (at - r * per));
}

// A map may not come about (a wait that ran out); the launches behind it are queued by then.  So behind B and M a segment's rows hold whether both are there, [0] B, [1] M,
// as MAPS found, and [2] whether the state before the segment can be, as FOLD concludes.  (The chunk that least_chunks adds has at least one token: room enough.)
constexpr int32_t IS_THERE = 0x7e571;
template <typename T>
__device__ __forceinline__ int32_t* there(const DeltaArgs& a, long long row, int hv) {
    return reinterpret_cast<int32_t*>(scratch<T>(a, row, hv, (a.dv + a.dk) * a.dk));
}

template <int D, typename T, int PHASE>
__global__ void __launch_bounds__(Shape<D, T>::THREADS, 1) delta_chunk_kernel(const DeltaArgs a) {
    using Z = Shape<D, T>;
    constexpr int KB = Z::KB, PARTS = Z::PARTS, KS = (D < 64 ? D : 64) / 16;        // K steps of 16 per block of 64
    constexpr int JOIN = D == 128 ? 2 : 8;                                          // see rows8
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* t_ring = smem + Z::K_STAGES * Z::KQ_BYTES;
    uint8_t* p_ring = t_ring + Z::T_STAGES * TRI_BYTES;
    uint8_t* prep_s = p_ring + Z::P_STAGES * TRI_BYTES;                             // per preparing team: matrix, scratch
    T* v_s = reinterpret_cast<T*>(prep_s + Z::PREPS * (Z::A_BYTES + Z::X_BYTES));   // [token][row]
    uint16_t* o_s = reinterpret_cast<uint16_t*>(reinterpret_cast<uint8_t*>(v_s) + Z::V_BYTES);       // [token][row]
    float* kco_s = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(o_s) + Z::O_BYTES);
    float* tco_s = kco_s + Z::K_STAGES * Z::KCO;
    float* tok_s = tco_s + Z::P_STAGES * Z::TCO;                                    // per preparing team: what undoes the tile rows' scales [128], alpha, g_C / g, beta
    float* max_s = tok_s + Z::PREPS * (128 + 3 * C);                                // [2][GROUPS][ROWS] largest of a row's part: S; D as weighted
    float* inv_s = max_s + 2 * Z::GROUPS * ROWS;                                    // [2][ROWS] what undoes the scales of S rows
    uint64_t* bars = reinterpret_cast<uint64_t*>(inv_s + 2 * ROWS);
    auto bar_k = [&](int i) { return smem_u32(bars + i % Z::K_STAGES); };           // keys, queries, their weights
    auto bar_kfree = [&](int i) { return smem_u32(bars + 3 + i % Z::K_STAGES); };
    // T and P: the barriers of even and odd chunks, however many tiles there are (a wait by parity does not tell a chunk's turn from the
    // one after next, and a team that comes early would take the one before for its own)
    auto bar_t = [&](int i) { return smem_u32(bars + 6 + (i & 1)); };
    auto bar_tfree = [&](int i) { return smem_u32(bars + 8 + (i & 1)); };           // T read, P read
    auto bar_pfree = [&](int i) { return smem_u32(bars + 19 + (i & 1)); };
    auto k_turn = [](int i) { return (uint32_t)(i / Z::K_STAGES) & 1; };
    auto t_turn = [](int i) { return (uint32_t)(i >> 1) & 1; };
    const uint32_t bar_v = smem_u32(bars + 10), bar_vfree = smem_u32(bars + 11);    // values
    const uint32_t bar_z = smem_u32(bars + 12), bar_d = smem_u32(bars + 13), bar_s = smem_u32(bars + 14), bar_o = smem_u32(bars + 15);      // MMA sets
    const uint32_t bar_ofree = smem_u32(bars + 16);                                 // the outputs' accumulators read out
    auto bar_prep = [&](int w) { return smem_u32(bars + 17 + w); };
    const uint32_t bar_acc = smem_u32(bars + 21);                                   // a team has read its products out (ONE_ACC)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 22);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int hv = blockIdx.y, hk = hv / (a.Hv / a.Hk), row_base = blockIdx.x * ROWS;
    // MAPS: B of segments 0 .. P - 2, then M of 1 .. P - 2; OUTPUTS: segments 0 .. P - 1
    const int parts = PHASE == WHOLE ? 1 : PHASE == MAPS ? 2 * a.segments - 3 : a.segments, sequence = blockIdx.z / parts, part = blockIdx.z % parts;
    const bool identity = PHASE == MAPS && part >= a.segments - 1, first_cta = blockIdx.x == 0 && hv == 0 && part == 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    Sequence seq = read_sequence(a, sequence, first_cta);
    if (!seq.live) return;                                                          // (the whole CTA)
    if (__syncthreads_or(taken_before(a, sequence, seq, tid, Z::THREADS))) {
        if (first_cta && tid == 0) report_taken(a, sequence);
        return;
    }
    const Segment seg = segment_of(seq.length, identity ? part - a.segments + 2 : part, PHASE == WHOLE ? 1 : a.segments, D, a.dv, (int)sizeof(T));
    if (seg.count == 1 ? PHASE == MAPS || seg.p > 0 : identity && blockIdx.x > 0) return;
    seq.begin += seg.begin;
    seq.length = seg.length;
    if (PHASE == OUTPUTS && seg.p > 0 && there<T>(a, seq.begin, hv)[2] != IS_THERE) return;     // (reported by MAPS; the state stays as it is)
    const int n = (seq.length + C - 1) / C;                                         // chunks
    if (tid == 0) {
        for (int s = 0; s < 3; ++s) {
            mbar_init(smem_u32(bars + s), 128);                                     // the preparing threads
            mbar_init(smem_u32(bars + 3 + s), 1 + 128);                             // the chain's commit, the output threads
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(bars + 6 + s), 128);
            mbar_init(smem_u32(bars + 8 + s), 1);
            mbar_init(smem_u32(bars + 19 + s), 1);
        }
        mbar_init(bar_acc, 128);
        mbar_init(bar_v, 128);
        mbar_init(bar_vfree, 1);
        mbar_init(bar_z, 1);
        mbar_init(bar_d, 1);
        mbar_init(bar_s, 1);
        mbar_init(bar_o, 2);                                                        // the commit, and the chain's leader (scales of the rows)
        mbar_init(bar_ofree, 128);
        for (int w = 0; w < 2; ++w) mbar_init(bar_prep(w), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(Z::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    // (not before tensor memory is this CTA's: a dependent launch may hold some of it while it waits for this one)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    bool fail = false;
    // MMAs complete by themselves: nobody gives up early and leaves them behind
    auto wait_mma = [&](uint32_t bar, uint32_t parity) {
        if (!sm100::mbar_wait(bar, parity)) {
            fail = true;
            *abort_flag = 1;
        }
    };
    // what another role has to do: bounded, and given up as soon as a role has
    auto wait = [&](uint32_t bar, uint32_t parity) {
        for (int i = 0; i < sm100::WAIT_LIMIT; ++i) {
            if (sm100::mbar_try_wait(bar, parity)) return;
            if ((i & 63) == 63 && *abort_flag) break;
        }
        fail = true;
        *abort_flag = 1;
    };

    if (warp < 4 * Z::PREPS) {
        // =============================== PREPARATION ===============================
        if constexpr (Z::SPLIT_REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Z::PREP_REGS));
        const int team = warp >> 2, w4 = warp & 3, pt = tid & 127;
        float* A_s = reinterpret_cast<float*>(prep_s + team * (Z::A_BYTES + Z::X_BYTES));       // [C][AP]
        float* X_s = A_s + Z::A_BYTES / 4;                                                      // [32][36]
        float* scale_s = tok_s + team * (128 + 3 * C);
        float *alpha_s = scale_s + 128, *behind_s = alpha_s + C, *total_s = behind_s + C;       // total_s: product of the gates of either warp
        const uint32_t acc_at = uniform(tmem_base + Z::PREP_COL + (Z::ONE_ACC ? 0 : team * C));
        constexpr int VEC = Vec16<T>::N, CPR = D / VEC, LR = CPR < 8 ? CPR : 8;      // 16-byte chunks and lanes per row
        constexpr int PASS_ROWS = 128 / LR, PASSES = 128 / PASS_ROWS, NC = CPR / LR;
        constexpr int BATCH = PASSES * NC > 4 ? 4 / NC : PASSES;                     // passes whose loads are in flight together
        const T* kp = static_cast<const T*>(a.k) + seq.begin * a.k_stride + (long long)hk * D;
        const T* qp = static_cast<const T*>(a.q) + seq.begin * a.q_stride + (long long)hk * D;
        auto gate_of = [&](const float* g, int t, float pad) { return t < seq.length ? __ldg(g + (seq.begin + t) * a.gate_stride + hv) : pad; };
        float alpha_next = 1.f, beta_next = 0.f;
        if (team < n && pt < C) {
            alpha_next = gate_of(a.alpha, team * C + pt, 1.f);
            beta_next = gate_of(a.beta, team * C + pt, 0.f);
        }
        auto products_read = [&] {                                                  // (their place is the other team's next)
            if (Z::ONE_ACC) {
                tc_fence_before();
                arrive(bar_acc);
            }
        };
        uint32_t phase = 0;
        for (int i = team; i < n; i += Z::PREPS) {
            const int t0 = i * C;
            uint8_t* KQ_s = smem + i % Z::K_STAGES * Z::KQ_BYTES;
            float* kco = kco_s + i % Z::K_STAGES * Z::KCO;
            if (i >= Z::K_STAGES) wait(bar_kfree(i), k_turn(i - Z::K_STAGES));
            // keys (rows 0 - 63) and queries (64 - 127) as the K-major operand tile, every row with its own power of two; tokens
            // beyond the sequence are zeros with alpha = 1, beta = 0: they change nothing
            const int lr = pt % LR, row0 = pt / LR;
#pragma unroll 1
            for (int p0 = 0; p0 < PASSES; p0 += BATCH) {
                uint4 raw[BATCH][NC];
#pragma unroll
                for (int p = 0; p < BATCH; ++p) {
                    const int row = (p0 + p) * PASS_ROWS + row0, t = t0 + (row & 63);
                    const T* src = row < C ? kp + t * a.k_stride : qp + t * a.q_stride;
#pragma unroll
                    for (int c = 0; c < NC; ++c) raw[p][c] = t < seq.length ? __ldg(reinterpret_cast<const uint4*>(src) + c * LR + lr) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int p = 0; p < BATCH; ++p) {
                    const int row = (p0 + p) * PASS_ROWS + row0;
                    float x[NC * VEC], m = 0.f;
#pragma unroll
                    for (int c = 0; c < NC; ++c) Vec16<T>::unpack(raw[p][c], x + c * VEC);
#pragma unroll
                    for (int e = 0; e < NC * VEC; e += 2) m = max3(m, x[e], x[e + 1]);
#pragma unroll
                    for (int o = LR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                    float sc, inv;
                    pow2_scale(m, NARROW, sc, inv);
#pragma unroll
                    for (int e = 0; e < NC * VEC; e += 2) {
                        const float2 y = __fmul2_rn(pair(x[e], x[e + 1]), pair(sc, sc));
                        x[e] = y.x;
                        x[e + 1] = y.y;
                    }
                    if (lr == 0) scale_s[row] = m > 0x1p-122f ? inv : 0.f;     // (below that the row is nothing in fp16: so is what it undoes)
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const int el = (c * LR + lr) * VEC;
                        uint8_t* dst = KQ_s + (el >> 6) * KQ_BLOCK + row * 128 + ((((el & 63) >> 3) ^ (row & 7)) << 4) + (el & 7) * 2;
                        const float* y = x + c * VEC;
                        if constexpr (VEC == 8) {        // bf16: exact in one fp16 number
                            *reinterpret_cast<uint4*>(dst) = make_uint4(pack_f16x2(y[0], y[1]), pack_f16x2(y[2], y[3]), pack_f16x2(y[4], y[5]), pack_f16x2(y[6], y[7]));
                        } else {
                            uint32_t hi[2], lo[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) split2(y[2 * e], y[2 * e + 1], hi[e], lo[e]);
                            *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0], hi[1]);
                            *reinterpret_cast<uint2*>(dst + KB * KQ_BLOCK) = make_uint2(lo[0], lo[1]);
                        }
                    }
                }
            }
            // products of the gates: up to a token (g) and behind it
            float g = alpha_next, behind = alpha_next;
            const float beta = beta_next;
            if (pt < C) {
                alpha_s[pt] = alpha_next;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const float x = __shfl_up_sync(0xffffffffu, g, o), y = __shfl_down_sync(0xffffffffu, behind, o);
                    if (lane >= o) g *= x;
                    if (lane + o < 32) behind *= y;
                }
                if (lane == 0) total_s[w4] = behind;
                behind = __shfl_down_sync(0xffffffffu, behind, 1);
                if (lane == 31) behind = 1.f;
                if (i + Z::PREPS < n) {
                    alpha_next = gate_of(a.alpha, t0 + Z::PREPS * C + pt, 1.f);
                    beta_next = gate_of(a.beta, t0 + Z::PREPS * C + pt, 0.f);
                }
            }
            if (Z::ONE_ACC && i > 0) wait(bar_acc, (i - 1) & 1);
            proxy_fence();
            tc_fence_before();
            if (bar_or(1 + team, 128, fail ? 1 : 0)) { fail = true; break; }
            if (w4 == 0) {          // [K; Q] K^T
                tc_fence_after();
                const uint64_t kd = umma_desc(uniform(smem_u32(KQ_s)));
#pragma unroll 1
                for (int t = PARTS > 1 ? 2 : 0; t >= 0; --t)                // small terms first: (lo hi, hi lo,) hi hi
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            const int at = (kb * KQ_BLOCK + ks * 32) >> 4, low = (KB * KQ_BLOCK) >> 4;
                            mma_ss(acc_at, kd + (at + (t == 2 ? low : 0)), kd + (at + (t == 1 ? low : 0)), idesc_f16(C), t != (PARTS > 1 ? 2 : 0) || kb || ks);
                        }
                mma_commit(bar_prep(team));
            }
            if (pt < C) {
                if (w4 == 1) g *= total_s[0];
                else behind *= total_s[1];
                kco[pt] = beta * (g * scale_s[pt]);
                kco[C + pt] = g * scale_s[C + pt];
                kco[2 * C + pt] = beta;
                if (pt == C - 1) kco[3 * C] = g;
                behind_s[pt] = behind * scale_s[pt];                            // (and what undoes the key's scale)
            }
            arrive(bar_k(i));
            if (i + Z::PREPS < n) { // the lines of the team's next chunk into L2
                constexpr int LINES = D * (int)sizeof(T) / 128 > 0 ? D * (int)sizeof(T) / 128 : 1;
                for (int x = pt; x < 2 * C * LINES; x += 128) {
                    const int row = (x >> 1) / LINES, ln = (x >> 1) % LINES, t = min(t0 + Z::PREPS * C + row, seq.length - 1);
                    const char* p = reinterpret_cast<const char*>((x & 1) ? qp + t * a.q_stride : kp + t * a.k_stride) + ln * 128;
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
                }
            }
            wait_mma(bar_prep(team), phase);
            phase ^= 1;
            tc_fence_after();
            // A's row i by thread i, P's row i by thread 64 + i.  (g_i / g_l) runs from the right: the product of the gates behind l.
            uint8_t *T_s = t_ring + i % Z::T_STAGES * TRI_BYTES, *P_s = p_ring + i % Z::P_STAGES * TRI_BYTES;
            float* tco = tco_s + i % Z::P_STAGES * Z::TCO;
            if (w4 < 2) {
                const float coef = beta * scale_s[pt];
                float ratio = 1.f;
#pragma unroll 1
                for (int cb = 3; cb >= 0; --cb) {
                    uint32_t v[16];
                    tmem_ld16(acc_at + cb * 16 + ((uint32_t)(w4 * 32) << 16), v);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 12; e >= 0; e -= 4) {
                        const float4 al = *reinterpret_cast<const float4*>(alpha_s + cb * 16 + e), ki = *reinterpret_cast<const float4*>(scale_s + cb * 16 + e);
                        const float alv[4] = {al.x, al.y, al.z, al.w}, kiv[4] = {ki.x, ki.y, ki.z, ki.w};
                        float row[4];
#pragma unroll
                        for (int f = 3; f >= 0; --f) {
                            const int l = cb * 16 + e + f;
                            row[f] = l < pt ? (coef * ratio) * (__uint_as_float(v[e + f]) * kiv[f]) : 0.f;
                            ratio *= l <= pt ? alv[f] : 1.f;
                        }
                        *reinterpret_cast<float4*>(A_s + pt * AP + cb * 16 + e) = make_float4(row[0], row[1], row[2], row[3]);
                    }
                }
                products_read();
                __syncwarp();
                // T = (I + A)^-1 in place, from the diagonal out.  Blocks of 16, two per warp, one column per lane by forward
                // substitution; then a warp's two blocks are joined, then the two warps': - T22 A21 T11 below the diagonal.
                float* L = A_s + (w4 * 32) * (AP + 1) + (lane >> 4) * (16 * AP + 16);
                const int col = lane & 15;
                float x[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float s0 = r == col ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
                    for (int l = 0; l < r; l += 4) {
                        const float4 q = *reinterpret_cast<const float4*>(L + r * AP + l);
                        s0 = fmaf(-q.x, x[l], s0);
                        if (l + 1 < r) s1 = fmaf(-q.y, x[l + 1], s1);
                        if (l + 2 < r) s0 = fmaf(-q.z, x[l + 2], s0);
                        if (l + 3 < r) s1 = fmaf(-q.w, x[l + 3], s1);
                    }
                    x[r] = s0 + s1;
                }
                __syncwarp();
#pragma unroll
                for (int r = 0; r < 16; ++r) L[r * AP + col] = x[r];
                __syncwarp();
                float* B21 = A_s + (w4 * 32) * (AP + 1) + (16 + (lane >> 4) * 8) * AP;       // eight rows of the lower block per half warp
                float acc[8];
                rows8<16, JOIN>(acc, B21, A_s + (w4 * 32) * (AP + 1) + col, AP);
#pragma unroll
                for (int r = 0; r < 8; ++r) X_s[w4 * (16 * 20) + ((lane >> 4) * 8 + r) * 20 + col] = acc[r];
                __syncwarp();
                rows8<16, JOIN>(acc, B21 + 16, X_s + w4 * (16 * 20) + col, 20);
                __syncwarp();
#pragma unroll
                for (int r = 0; r < 8; ++r) B21[r * AP + col] = -acc[r];
            } else {
                const int me = pt - C;
                const float query = scale_s[pt];
                float ratio = 1.f;
                if (i >= Z::P_STAGES) wait(bar_pfree(i - Z::P_STAGES), t_turn(i - Z::P_STAGES));
#pragma unroll 1
                for (int cb = 3; cb >= 0; --cb) {
                    uint32_t v[16];
                    tmem_ld16(acc_at + cb * 16 + ((uint32_t)(w4 * 32) << 16), v);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 12; e >= 0; e -= 4) {
                        const float4 al = *reinterpret_cast<const float4*>(alpha_s + cb * 16 + e), ki = *reinterpret_cast<const float4*>(scale_s + cb * 16 + e);
                        const float alv[4] = {al.x, al.y, al.z, al.w}, kiv[4] = {ki.x, ki.y, ki.z, ki.w};
#pragma unroll
                        for (int f = 3; f >= 0; --f) {
                            const int l = cb * 16 + e + f;
                            const float x = (__uint_as_float(v[e + f]) * kiv[f]) * query;
                            v[e + f] = __float_as_uint(l <= me ? ratio * x : 0.f);
                            ratio *= l <= me ? alv[f] : 1.f;
                        }
                    }
                    if (me >= 16 * cb) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) store_tri(P_s, me, cb, e, v + 8 * e);
                    }
                }
                products_read();
            }
            tc_fence_before();
            bar_or(1 + team, 128, 0);
            {
                float acc[8];
                rows8<32, JOIN>(acc, A_s + (32 + 8 * w4) * AP, A_s + lane, AP);
#pragma unroll
                for (int r = 0; r < 8; ++r) X_s[(8 * w4 + r) * 36 + lane] = acc[r];
                bar_or(1 + team, 128, 0);
                rows8<32, JOIN>(acc, A_s + (32 + 8 * w4) * AP + 32, X_s + lane, 36);
#pragma unroll
                for (int r = 0; r < 8; ++r) A_s[(32 + 8 * w4 + r) * AP + lane] = -acc[r];
            }
            if (i >= Z::T_STAGES) wait(bar_tfree(i - Z::T_STAGES), t_turn(i - Z::T_STAGES));
            if (bar_or(1 + team, 128, fail ? 1 : 0)) { fail = true; break; }
            // T as an operand tile: row pt / 2 by threads pt and pt + 1, columns 16 h .. and 32 + 16 h .. (conflict-free reads).  (What lies above the
            // diagonal is zero, A's there too.)
            {
                const int ti = pt >> 1, hf = pt & 1;
#pragma unroll
                for (int c = 0; c < 4; ++c) {                               // chunks of eight columns
                    const int step = 2 * (c >> 1) + hf, half = c & 1;
                    if (ti < 16 * step) continue;
                    const float4 x = *reinterpret_cast<const float4*>(A_s + ti * AP + 16 * step + 8 * half), y = *reinterpret_cast<const float4*>(A_s + ti * AP + 16 * step + 8 * half + 4);
                    const uint32_t t[8] = {__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z), __float_as_uint(x.w),
                                           __float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z), __float_as_uint(y.w)};
                    store_tri(T_s, ti, step, half, t);
                }
                if (hf == 0) tco[ti] = behind_s[ti];
            }
            proxy_fence();
            arrive(bar_t(i));
        }
    } else if (warp < 4 * (Z::PREPS + Z::GROUPS)) {
        // =============================== STATE ROWS ===============================
        if constexpr (Z::SPLIT_REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Z::CHAIN_REGS));
        constexpr int G = Z::GROUPS, H = D / G, HB = H / 16, TG = C / G, TB = TG / 16;      // a thread's part of its row and of the tokens, in blocks of 16
        const int c = (warp >> 2) - Z::PREPS, r = (warp & 3) * 32 + lane;
        const bool is_row = identity ? r < D : row_base + r < a.dv;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem_base + lanes + c * H, z_at = tmem_base + lanes + Z::Z_COL + TG * c, d_at = tmem_base + lanes + Z::D_COL + TG * c;
        const uint32_t x_at = tmem_base + lanes + TB * c * Z::X_STEP, do_at = x_at + Z::DO_COL;
        const bool issuer = warp == 4 * Z::PREPS, leader = issuer && lane == 0;
        // largest magnitudes (kind 0: S; 1: D as weighted): mine, and of the whole row when all have met
        float* mine = max_s + c * ROWS + r;
        auto of_row = [&](int kind) {
            const float* m = max_s + kind * G * ROWS + r;
            float x = fmaxf(m[0], m[ROWS]);
#pragma unroll
            for (int e = 2; e < G; ++e) x = fmaxf(x, m[e * ROWS]);
            return x;
        };
        float* state = a.states + seq.slot * a.state_stride + ((long long)hv * a.dv + row_base + r) * D + c * H;
        auto meet = [&] { return bar_or(CHAIN_BARRIER, Z::CHAIN_THREADS, fail ? 1 : 0); };
        // the row's part, times 2^e; inv_row, scale_row: 2^-e, 2^e.  The exponent changes only when the row's largest element leaves a
        // window in which two fp16 parts hold it to 22 bits.
        float S[H], m = 0.f, inv_row = 1.f, scale_row = 1.f;
#pragma unroll
        for (int e = 0; e < H; e += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (PHASE == OUTPUTS && seg.count > 1) {
                if (is_row) x = __ldcs(scratch<T>(a, seq.begin, hv, (row_base + r) * D + c * H + e));
            } else if (identity) {
                const int at = c * H + e;
                x = make_float4(r == at, r == at + 1, r == at + 2, r == at + 3);
            } else if (is_row && !seq.fresh && seg.p == 0) {
                x = __ldcs(reinterpret_cast<const float4*>(state + e));
            }
            S[e] = x.x; S[e + 1] = x.y; S[e + 2] = x.z; S[e + 3] = x.w;
        }
#pragma unroll
        for (int e = 0; e < H; e += 2) m = max3(m, S[e], S[e + 1]);
        if (PHASE == MAPS && seg.p == 0 && is_row) {              // (OUTPUTS' last segment may be done with the state before its first one begins)
#pragma unroll
            for (int e = 0; e < H; e += 4) *scratch<T>(a, seq.begin, hv, (row_base + r) * D + c * H + e) = make_float4(S[e], S[e + 1], S[e + 2], S[e + 3]);
        }
        *mine = m;
        meet();
        int issued = 0;                                           // chunks whose last products have been issued
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const uint32_t turn = i & 1;
            const float* kco = kco_s + i % Z::K_STAGES * Z::KCO;
            const float* tco = tco_s + i % Z::P_STAGES * Z::TCO;
            // ---- Z = S K^T, and S Q^T ----
            m = of_row(0);
            if (!(m < 0x1p15f) || (m < 0x1p6f && m > 0.f && scale_row < 0x1p110f)) {
                float sc, inv;
                pow2_scale(m, WIDE, sc, inv);
                if (sc > 0x1p110f * inv_row) {                    // (what undoes it, in products with D too, stays a normal number: a state below 2^-110 loses places)
                    sc = 0x1p110f * inv_row;
                    inv = 0x1p-110f * scale_row;
                }
#pragma unroll
                for (int e = 0; e < H; e += 2) {
                    const float2 y = __fmul2_rn(pair(S[e], S[e + 1]), pair(sc, sc));
                    S[e] = y.x;
                    S[e + 1] = y.y;
                }
                inv_row *= inv;
                scale_row *= sc;
            }
            __syncwarp();
#pragma unroll
            for (int b = 0; b < HB; ++b) split_to_tmem(s_at + 16 * b, S + 16 * b);
            if (c == 0) inv_s[turn * ROWS + r] = inv_row;
            tc_wait_st();
            tc_fence_before();
            wait(bar_k(i), k_turn(i));
            if (i > 0) wait(bar_ofree, turn ^ 1);
            if (meet()) { fail = true; break; }
            if (issuer) {
                tc_fence_after();
                const uint64_t kd = umma_desc(uniform(smem_u32(smem + i % Z::K_STAGES * Z::KQ_BYTES)));
                bool first = true;
                auto product = [&](int sp, int kp) {
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const int kb = ks / KS;
                        mma_ts(tmem_base + Z::Z_COL, tmem_base + ks * 16 + sp * 8, kd + ((((kp * KB + kb) * KQ_BLOCK) + (ks - kb * KS) * 32) >> 4), idesc_f16(2 * C), !first);
                        first = false;
                    }
                };
                product(1, 0);
                if constexpr (PARTS > 1) product(0, 1);
                product(0, 0);
                mma_commit(bar_z);
            }
            float val[Z::STAGE_V ? 1 : TG];                       // fp32 values: from global memory, beside the product
            if constexpr (Z::STAGE_V) {
                wait(bar_v, turn);
            } else {
                const T* vp = static_cast<const T*>(a.v) + seq.begin * a.v_stride + (long long)hv * a.dv + row_base + r;
#pragma unroll
                for (int e = 0; e < TG; ++e) {
                    const int t = i * C + TG * c + e;
                    val[e] = is_row && !identity && t < seq.length ? __ldg(reinterpret_cast<const float*>(vp + t * a.v_stride)) : 0.f;
                }
            }
            wait_mma(bar_z, turn);
            tc_fence_after();
            // ---- X = (V^T - Z diag(g)) diag(beta), over the S operand (read by now) ----
            float x[TG];
            const float2 neg = pair(-inv_row, -inv_row);
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                uint32_t v[16];
                tmem_ld16(z_at + 16 * b, v);
                float u[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if constexpr (Z::STAGE_V) u[e] = __bfloat162float(v_s[(TG * c + 16 * b + e) * ROWS + r]);
                    else u[e] = val[16 * b + e];
                }
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 gz = *reinterpret_cast<const float4*>(kco + TG * c + 16 * b + e), be = *reinterpret_cast<const float4*>(kco + 2 * C + TG * c + 16 * b + e);
                    const float2 y0 = __ffma2_rn(__fmul2_rn(pair(v[e], v[e + 1]), neg), pair(gz.x, gz.y), __fmul2_rn(pair(u[e], u[e + 1]), pair(be.x, be.y)));
                    const float2 y1 = __ffma2_rn(__fmul2_rn(pair(v[e + 2], v[e + 3]), neg), pair(gz.z, gz.w), __fmul2_rn(pair(u[e + 2], u[e + 3]), pair(be.z, be.w)));
                    x[16 * b + e] = y0.x; x[16 * b + e + 1] = y0.y; x[16 * b + e + 2] = y1.x; x[16 * b + e + 3] = y1.y;
                }
                triple_to_tmem(x_at + Z::X_STEP * b, x + 16 * b);
            }
            const float g_chunk = kco[3 * C];
            tc_wait_st();
            tc_fence_before();
            wait(bar_t(i), t_turn(i));
            if (meet()) { fail = true; break; }
            if (Z::STAGE_V && leader) arrive(bar_vfree);
            // T's or P's products, an operand in three parts on either side: what is below 2^-24 of the largest left out, small terms first
            auto triangle = [&](uint32_t to, uint32_t from, const uint8_t* tile) {
                const uint64_t at = tri_desc(uniform(smem_u32(tile)));
                constexpr int PART[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
#pragma unroll
                for (int t = 0; t < 6; ++t)
#pragma unroll
                    for (int ks = 0; ks < C / 16; ++ks)
                        mma_ts(tmem_base + to + 16 * ks, tmem_base + from + Z::X_STEP * ks + 8 * PART[t][0], at + tri_step(ks) + ((PART[t][1] * TRI) >> 4),
                               idesc_f16(C - 16 * ks) | BF16_OPERANDS, t != 0 || ks != 0);
            };
            // ---- D = X T^T ----
            if (issuer) {
                tc_fence_after();
                triangle(Z::D_COL, 0, t_ring + i % Z::T_STAGES * TRI_BYTES);
                mma_commit(bar_d);
                mma_commit(bar_tfree(i));
            }
            wait_mma(bar_d, turn);
            tc_fence_after();
            // ---- D's operand for the state: times g_C / g (and what undoes the keys' scales) ----
            float me = 0.f;
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                uint32_t v[16];
                tmem_ld16(d_at + 16 * b, v);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 w = *reinterpret_cast<const float4*>(tco + TG * c + 16 * b + e);
                    const float2 d0 = pair(v[e], v[e + 1]), d1 = pair(v[e + 2], v[e + 3]), e0 = __fmul2_rn(d0, pair(w.x, w.y)), e1 = __fmul2_rn(d1, pair(w.z, w.w));
                    x[16 * b + e] = d0.x; x[16 * b + e + 1] = d0.y; x[16 * b + e + 2] = d1.x; x[16 * b + e + 3] = d1.y;
                    me = max3(max3(me, e0.x, e0.y), e1.x, e1.y);
                }
            }
            mine[G * ROWS] = me;
            if (meet()) { fail = true; break; }
            float inv_e, sc_e;
            pow2_scale(of_row(1), WIDE, sc_e, inv_e);
            // the row's old part and what is added, in the units of the new one; where either would leave fp32's range in the old units (gates far beyond
            // 1, values far above the state), smaller units
            float keep = g_chunk;
            if (fabsf(g_chunk) > 0x1p60f || (inv_e * 0x1p-64f) * (scale_row * 0x1p-64f) > 0x1p-68f) {
                float down, up;
                pow2_scale(fmaxf(fabsf(g_chunk), 1.f), 0, down, up);
                const float scale_new = fmaxf(fminf(scale_row * down, sc_e), 0x1p-120f);
                keep *= scale_new * inv_row;
                inv_row = __uint_as_float((254u << 23) - __float_as_uint(scale_new));      // 1 / a power of two
                scale_row = scale_new;
            }
            const float back = inv_e * scale_row;
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                float y[16];
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 w = *reinterpret_cast<const float4*>(tco + TG * c + 16 * b + e);
                    const float2 e0 = __fmul2_rn(pair(x[16 * b + e], x[16 * b + e + 1]), pair(w.x, w.y)), e1 = __fmul2_rn(pair(x[16 * b + e + 2], x[16 * b + e + 3]), pair(w.z, w.w));
                    y[e] = e0.x; y[e + 1] = e0.y; y[e + 2] = e1.x; y[e + 3] = e1.y;
                }
                split_to_tmem(d_at + 16 * b, y, sc_e);
            }
            tc_wait_st();
            tc_fence_before();
            if (meet()) { fail = true; break; }
            // ---- D K over the X operand (read by now); D's operand for the outputs meanwhile, and D P^T ----
            if (issuer) {
                tc_fence_after();
                const uint64_t kd = umma_desc_mn(uniform(smem_u32(smem + i % Z::K_STAGES * Z::KQ_BYTES)), KQ_BLOCK);
                bool first = true;
                auto product = [&](int dp, int kp) {
#pragma unroll
                    for (int ks = 0; ks < C / 16; ++ks) {
                        mma_ts(tmem_base, tmem_base + Z::D_COL + ks * 16 + dp * 8, kd + ((kp * KB * KQ_BLOCK + ks * 2048) >> 4), idesc_f16(D) | B_MN_MAJOR, !first);
                        first = false;
                    }
                };
                if constexpr (PARTS > 1) product(0, 1);
                product(1, 0);
                product(0, 0);
                mma_commit(bar_s);
            }
#pragma unroll
            for (int b = 0; b < TB; ++b) triple_to_tmem(do_at + Z::X_STEP * b, x + 16 * b);
            tc_wait_st();
            tc_fence_before();
            meet();                                                   // (nobody has waited since the last one: nobody gives up here)
            if (issuer) {
                tc_fence_after();
                triangle(Z::O2_COL, Z::DO_COL, p_ring + i % Z::P_STAGES * TRI_BYTES);
                mma_commit(bar_o);
                mma_commit(bar_kfree(i));
                mma_commit(bar_pfree(i));
            }
            if (leader) arrive(bar_o);
            issued = i + 1;
            wait_mma(bar_s, turn);
            tc_fence_after();
            m = 0.f;
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                uint32_t v[16];
                tmem_ld16(s_at + 16 * b, v);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 y2 = __ffma2_rn(pair(keep, keep), pair(S[16 * b + e], S[16 * b + e + 1]), __fmul2_rn(pair(v[e], v[e + 1]), pair(back, back)));
                    S[16 * b + e] = y2.x;
                    S[16 * b + e + 1] = y2.y;
                    m = max3(m, y2.x, y2.y);
                }
            }
            *mine = m;
            tc_fence_before();
            if (meet()) { fail = true; break; }
        }
#ifdef ONELA_TEST_HOOKS
        if (PHASE == MAPS && g_hook_delta_map_fails == 1 + part && sequence == 0 && hv == 0) fail = true;
#endif
        const bool come = !fail;                                  // (the same in all of the chain's threads, who have met since they last waited for what S needs)
        if (issued > 0) wait_mma(bar_o, (issued - 1) & 1);        // (the outputs' products too are over when tensor memory is freed)
        const bool last = PHASE == OUTPUTS && seg.p == seg.count - 1;
        if (PHASE == MAPS && leader) there<T>(a, seq.begin + seq.length, hv)[identity ? 1 : 0] = come ? IS_THERE : 0;
        if (come && is_row && (PHASE != OUTPUTS || last)) {
            const long long next_row = seq.begin + seq.length;    // of the next segment: where a map goes
            int to_at = (identity ? a.dv * D + r * D : (row_base + r) * D) + c * H;
            asm volatile("" : "+r"(to_at));                       // (not to be worked out ahead of the loop, which needs the registers)
#pragma unroll
            for (int e = 0; e < H; e += 4) {
                float4* to = reinterpret_cast<float4*>(state + e);
                if (PHASE == MAPS) to = scratch<T>(a, next_row, hv, to_at + e);
                *to = make_float4(S[e] * inv_row, S[e + 1] * inv_row, S[e + 2] * inv_row, S[e + 3] * inv_row);
            }
        }
    } else {
        // =============================== VALUES IN, OUTPUTS OUT ===============================
        if constexpr (Z::SPLIT_REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Z::OUT_REGS));
        const int ot = tid & 127, r = ot;
        const bool is_row = row_base + r < a.dv;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int rows = min(ROWS, a.dv - row_base);              // a multiple of 32
        const T* vp = static_cast<const T*>(a.v) + seq.begin * a.v_stride + (long long)hv * a.dv + row_base;
        T* out0 = static_cast<T*>(a.out) + seq.begin * a.out_stride + (long long)hv * a.dv + row_base;
        T* op = out0 + r;
        constexpr int VEC = Vec16<T>::N, CH = ROWS / VEC;         // 16-byte chunks per token
        const int v_token = ot / CH, v_chunk = ot % CH;           // this thread's of the first 128 / CH tokens
        const long long v_step = a.v_stride * (128 / CH), out_step = a.out_stride;
        auto load_values = [&](int i) {
            const T* from = vp + (long long)(i * C + v_token) * a.v_stride + v_chunk * VEC;
            uint32_t dst = smem_u32(v_s + v_token * ROWS + v_chunk * VEC);
            int left = v_chunk * VEC < rows && !identity ? seq.length - i * C - v_token : 0;
#pragma unroll 2
            for (int x = 0; x < C * CH / 128; ++x) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(left > 0 ? from : vp), "r"(left > 0 ? 16 : 0) : "memory");
                from += v_step;
                dst += 128 / CH * ROWS * (int)sizeof(T);
                left -= 128 / CH;
            }
            asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
            arrive(bar_v);
        };
#pragma unroll 1
        for (int i = -1; i < n && !fail; ++i) {                   // (-1: the first values only)
            const uint32_t turn = i & 1;
            const float* kco = kco_s + max(i, 0) % Z::K_STAGES * Z::KCO + C;
            if (Z::STAGE_V && i + 1 < n) {
                if (i >= 0) wait(bar_vfree, turn);
                if (!fail) load_values(i + 1);
            }
            if (!Z::STAGE_V && i + 1 < n) {                           // the lines of the next chunk's values into L2
                const int t = min((i + 1) * C + (ot >> 1), seq.length - 1);
                for (int x = (ot & 1) * 32; x < rows; x += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(vp + t * a.v_stride + x));
            }
            if (i < 0) continue;
            wait(bar_o, turn);
            if (bar_or(OUT_BARRIER, 128, fail ? 1 : 0)) { fail = true; break; }
            tc_fence_after();
            const float inv_row = inv_s[turn * ROWS + r];
            // read out first and stored behind that, so that the chain may go on (fp32: half of it, for want of registers)
            constexpr int PER = sizeof(T) == 2 ? 2 : 1, FIRST = PER == 2 ? 0 : 2;      // outputs per register; blocks of 16 stored at once
            T* dst = op + (long long)(i * C) * a.out_stride;
            const int left = is_row && PHASE != MAPS ? seq.length - i * C : 0;
            uint32_t o[(4 - FIRST) * 16 / PER];
            auto block = [&](int b, uint32_t* to) {
                uint32_t v[16], w[16];
                tmem_ld16(tmem_base + lanes + Z::O1_COL + 16 * b, v);
                tmem_ld16(tmem_base + lanes + Z::O2_COL + 16 * b, w);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 gq = *reinterpret_cast<const float2*>(kco + 16 * b + e);
                    const float2 y = __ffma2_rn(__fmul2_rn(pair(v[e], v[e + 1]), pair(inv_row, inv_row)), gq, pair(w[e], w[e + 1]));
                    if constexpr (PER == 2) {
                        to[e / 2] = sm100::pack_bf16x2(y.x, y.y);
                    } else {
                        to[e] = __float_as_uint(y.x);
                        to[e + 1] = __float_as_uint(y.y);
                    }
                }
            };
            auto store = [&](int first, int count, const uint32_t* from) {
#pragma unroll
                for (int e = 0; e < count; ++e) {
                    // (predicated, not branched around: a third of the code)
                    if constexpr (PER == 2)
                        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\t@p st.global.b16 [%0], %1;\n\t}" ::"l"(dst),
                                     "h"((uint16_t)(from[e / 2] >> (16 * (e & 1)))), "r"(first + e), "r"(left)
                                     : "memory");
                    else
                        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\t@p st.global.b32 [%0], %1;\n\t}" ::"l"(dst), "r"(from[e]), "r"(first + e), "r"(left)
                                     : "memory");
                    dst += out_step;
                }
            };
#pragma unroll 1
            for (int b = 0; b < FIRST; ++b) {
                block(b, o);
                store(16 * b, 16, o);
            }
#pragma unroll
            for (int b = FIRST; b < 4; ++b) block(b, o + (b - FIRST) * 16 / PER);
            tc_fence_before();
            arrive(bar_ofree);
            if constexpr (PER == 2) {
                // through shared memory: a thread has a row of the state, memory wants a token's rows side by side.  (Two bytes per thread and token
                // straight to memory were twice the code, and code is what limits two SMs that share an instruction cache.)
                const int there = PHASE == MAPS ? 0 : seq.length - i * C;
#pragma unroll
                for (int t0 = 0; t0 < C; t0 += Z::O_TOKENS) {
#pragma unroll
                    for (int e = 0; e < Z::O_TOKENS; ++e) o_s[e * ROWS + r] = (uint16_t)(o[(t0 + e) / 2] >> (16 * (e & 1)));
                    bar_or(OUT_BARRIER, 128, 0);
#pragma unroll 1
                    for (int x = ot; x < Z::O_TOKENS * ROWS / 8; x += 128) {
                        const int t = x / (ROWS / 8), ch = x % (ROWS / 8) * 8;
                        if (t0 + t < there && ch < rows)
                            *reinterpret_cast<uint4*>(out0 + (long long)(i * C + t0 + t) * a.out_stride + ch) = *reinterpret_cast<const uint4*>(o_s + t * ROWS + ch);
                    }
                    bar_or(OUT_BARRIER, 128, 0);
                }
            } else {
                store(16 * FIRST, C - 16 * FIRST, o);
            }
            arrive(bar_kfree(i));
        }
    }
    if (fail && a.status && atomicCAS(a.status, ONELA_OK, ONELA_E_TIMEOUT) == ONELA_OK) a.status[1] = sequence;
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(Z::TMEM_COLS) : "memory");
}

// The states before segments 2 .. P - 1 of a cut sequence: S <- S M_p + B_p, p = 1 .. P - 2, from the state before segment 1, each in the place of its B.  A
// CTA has 16 rows of the state, which need no others; S and M in shared memory, the next M on its way meanwhile, fp32 throughout.  (M read from
// global memory as it is used: 30 us a segment against 6.)
constexpr int FOLD_ROWS = 16, FOLD_THREADS = 256;
template <int D>
constexpr int fold_smem() { return (2 * D * D + FOLD_ROWS * D) * 4; }
template <int D, typename T>
__global__ void __launch_bounds__(FOLD_THREADS) delta_fold_kernel(const DeltaArgs a) {
    constexpr int GROUPS = FOLD_THREADS / D, OWN = FOLD_ROWS / GROUPS;              // threads per column; rows per thread
    extern __shared__ __align__(16) float fold_s[];
    float *M_s = fold_s, *S_s = fold_s + 2 * D * D;                                 // [2][D][D], [FOLD_ROWS][D]
    const int hv = blockIdx.y, row0 = blockIdx.x * FOLD_ROWS, col = threadIdx.x % D, own0 = threadIdx.x / D * OWN;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Sequence seq = read_sequence(a, blockIdx.z, false);
    if (!seq.live || __syncthreads_or(taken_before(a, blockIdx.z, seq, threadIdx.x, FOLD_THREADS))) return;
    if (segment_of(seq.length, 0, a.segments, D, a.dv, (int)sizeof(T)).count == 1) return;
    auto row_of = [&](int p) { return seq.begin + segment_of(seq.length, p, a.segments, D, a.dv, (int)sizeof(T)).begin; };
    auto fetch = [&](int p) {                                                       // M_p, which lies in the rows of segment p + 1
        const long long at = row_of(p + 1);
        for (int x = threadIdx.x; x < D * D / 4; x += FOLD_THREADS)
            sm100::cp_async16(smem_u32(M_s + (p & 1) * D * D + 4 * x), scratch<T>(a, at, hv, a.dv * D + 4 * x));
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (blockIdx.x == 0 && threadIdx.x < 32) {                                      // lane p: segment p
        const int p = threadIdx.x;
        int32_t* at = p > 0 && p < a.segments ? there<T>(a, row_of(p), hv) : nullptr;
        const uint32_t missing = __ballot_sync(0xffffffffu, at && (at[0] != IS_THERE || (p > 1 && at[1] != IS_THERE)));
        if (at) at[2] = missing << (31 - p) ? 0 : IS_THERE;
    }
    fetch(1);
    for (int x = threadIdx.x; x < FOLD_ROWS * D / 4; x += FOLD_THREADS)             // the state before segment 1
        *reinterpret_cast<float4*>(S_s + 4 * x) = *scratch<T>(a, row_of(1), hv, row0 * D + 4 * x);
    for (int p = 1; p + 1 < a.segments; ++p) {
        const long long at = row_of(p + 1);
        float acc[OWN];
        float* place[OWN];
#pragma unroll
        for (int r = 0; r < OWN; ++r) {
            const int e = (row0 + own0 + r) * D + col;
            place[r] = reinterpret_cast<float*>(scratch<T>(a, at, hv, e & ~3)) + (e & 3);
            acc[r] = *place[r];
        }
        if (p + 2 < a.segments) {
            fetch(p + 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        const float* M = M_s + (p & 1) * D * D + col;
#pragma unroll 4
        for (int k = 0; k < D; k += 4) {
            const float m0 = M[k * D], m1 = M[(k + 1) * D], m2 = M[(k + 2) * D], m3 = M[(k + 3) * D];
#pragma unroll
            for (int r = 0; r < OWN; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(S_s + (own0 + r) * D + k);
                acc[r] = fmaf(x.x, m0, fmaf(x.y, m1, fmaf(x.z, m2, fmaf(x.w, m3, acc[r]))));
            }
        }
        __syncthreads();                                                            // S has been read, and M, whose place the one after next takes
#pragma unroll
        for (int r = 0; r < OWN; ++r) {
            S_s[(own0 + r) * D + col] = acc[r];
            *place[r] = acc[r];
        }
    }
}

template <int D, typename T, int PHASE>
cudaError_t launch_phase(const DeltaArgs& a, int parts, cudaStream_t stream) {
    using Z = Shape<D, T>;
    auto kern = delta_chunk_kernel<D, T, PHASE>;
    constexpr int MAX_DEVICES = 64;
    static std::mutex setup_mutex;
    static bool ready[MAX_DEVICES] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(setup_mutex);
        if (!ready[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Z::SMEM);
            if (e != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    return launch_dependent(kern, dim3((a.dv + ROWS - 1) / ROWS, a.Hv, a.num_sequences * parts), dim3(Z::THREADS), Z::SMEM, stream, a);
}
template <int D, typename T>
cudaError_t launch_dt(const DeltaArgs& a, cudaStream_t stream) {
    if (a.segments == 1) return launch_phase<D, T, WHOLE>(a, 1, stream);
    cudaError_t e = cudaFuncSetAttribute(delta_fold_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, fold_smem<D>());
    if (e == cudaSuccess) e = launch_phase<D, T, MAPS>(a, 2 * a.segments - 3, stream);
    if (e == cudaSuccess)
        e = launch_dependent(delta_fold_kernel<D, T>, dim3(a.dv / FOLD_ROWS, a.Hv, a.num_sequences), dim3(FOLD_THREADS), fold_smem<D>(), stream, a);
    return e == cudaSuccess ? launch_phase<D, T, OUTPUTS>(a, a.segments, stream) : e;
}
template <int D>
cudaError_t launch_d(const DeltaArgs& a, int32_t dtype, cudaStream_t stream) {
    return dtype == ONELA_DTYPE_BF16 ? launch_dt<D, __nv_bfloat16>(a, stream) : launch_dt<D, float>(a, stream);
}

}  // namespace

#ifdef ONELA_TEST_HOOKS
extern "C" int onela_testhook_delta_map_fails(int part) { return (int)cudaMemcpyToSymbol(g_hook_delta_map_fails, &part, sizeof(int)); }
#endif

bool delta_chunk_supported(int32_t dk, int32_t) { return dk == 32 || dk == 64 || dk == 128; }

// Segments.  A chunk takes every CTA about the same time, whatever shares the GPU; one CTA fits an SM.  P segments of n chunks cost ceil(n / P) chunks twice,
// the fold a third of a chunk per segment and the launches about two; MAPS has 2 P - 3 CTAs per chain.
cudaError_t launch_delta_chunk(DeltaArgs a, int32_t dtype, long long longest, cudaStream_t stream) {
    constexpr int SMS = 148, MOST = 16;
    const long long chains = (long long)((a.dv + ROWS - 1) / ROWS) * a.Hv * a.num_sequences, chunks = (longest + C - 1) / C;
    double best = (double)chunks;
    // (one block of rows only: another one's outputs would overwrite what a state's second block has yet to read)
    for (int p = 3; p <= MOST && a.dv <= ROWS && chains * (2 * p - 3) <= SMS && chunks / p >= least_chunks(a.dk, a.dv, dtype == ONELA_DTYPE_BF16 ? 2 : 4); ++p) {
        const double cost = 2.0 * (double)((chunks + p - 1) / p) + (p - 2) / 3.0 + 3.0;
        if (cost < best) {
            best = cost;
            a.segments = p;
        }
    }
    return a.dk == 32 ? launch_d<32>(a, dtype, stream) : a.dk == 64 ? launch_d<64>(a, dtype, stream) : launch_d<128>(a, dtype, stream);
}

}  // namespace onela
