// Split-KV flash decoding of both paths over E4M3 pages with a scale per page and head, tokens on the MMA's M axis:
//
//   absorb path, Eq. (mqa) lines 3-5    x_t = scale s_t (q_hat . k8_t)                       o = sum_t p_t s_t k8_t[:512] / sum_t p_t
//   GQA path, Eq. (mha)                 x_t = scale (s^K_t (q_C . kC8_t) + s^R_t (q_R . kR8_t))  o = sum_t p_t s^V_t v8_t / sum_t p_t
//
//   S^T = K Q^T     M = 128 tokens, N = R query rows               (A = K tile, B = Q, both K-major)
//   O^T = V^T P^T   M = 128 value columns, N = 2 R, K = 128 tokens (A = V tile read MN-major, B = P^T rows)
//
// Queries and probabilities keep the precision of the bf16 path although the tensor core multiplies E4M3 by E4M3:
//   * A query row is scaled by a power of two to a maximum in (224, 448] and cut into two codes, q = hi + lo.  Four significant bits
//     each hold the eight of a bf16 value (the difference from the nearest hi is a multiple of the value's last bit and at most eight
//     of them), so the scores are those of the bf16 query as long as an element is not below 2^-15 of its row's largest;
//     what is smaller keeps an absolute error of 2^-19 of the largest.  Both terms' products go into one accumulator.
//   * With y_t = x_t + log2 s^V_t (log2 units), P'_t = 2^(y_t - m) is the token's weight with its V scale in it, which bounds what
//     P' has to represent to the token's share of the output.  P' is cut into hi and 16 lo, both E4M3, which multiply into columns
//     of their own: O = O_hi + O_lo / 16.  Relative error 2^-9 (hi leaves at most 2^-4 of a binade, lo rounds that to four
//     bits), absolute one 2^-14 where the reference puts the largest P' between 2^6 and 2^8.75: 2^-20 of a row's largest weight.
//     The sum over p = P' / s^V is taken in fp32 before any rounding.
// The tensor core does twice the method's products at E4M3 rate, i.e. what the bf16 path pays, on half the bytes.
//
//   * The softmax is that of tc_decode_gqa_t.cuh: a TMEM lane is a token, a thread has one token and eight query rows, every thread
//     holds its rows' references, and the four warps that share rows ask once per tile, in a barrier of their own, whether any score
//     outgrew its reference by more than kP8Grow binades.  The producer looks up the scales along with the rows and leaves them in
//     shared memory.
//   * R = 16 or 32 query rows per CTA.  More rows (64 heads of the absorb path, s_q > 1) are blocks of 32 on CTAs of their own
//     that walk the same tiles at the same time, so that the cache comes from HBM once and from L2 otherwise.  (Beyond 64 rows
//     absorb path calls of more pieces than workers here run on tc_decode_fp8_pair.cuh.)
//   * Measured, merge included, in a graph of 18 passes; in brackets calls one after another for longer, at the power cap.  Absorb path, 32
//     heads, 128 ragged sequences of up to 16384 rows: 127 us, 4.5 TB/s (142 to 149).  GQA path: 32 heads, 64 of up to 16384, 207 us, 5.5
//     TB/s, bound by HBM (213 to 224); 128 heads, s_q = 2, 64 of 4096, 130 us, 4.3 TB/s (143 to 150), with 45 % of the issue slots, 47 % of
//     DRAM and 13 % of the tensor pipe in use: bound by a tile's chain of waits (scores -> maximum -> weights -> P V).  In the same way the
//     absorb path's tile (25 %, 38 % and 16 %).  A chunk of 256 query positions over 2 x 4096 rows, 32 heads: absorb path 136 us on pairs
//     (1.08 PFLOP/s of the method's products), GQA path 146 us (0.29).
//   * Absorb path: V is the latent part of the K tile, which is read in both orders from one place in shared memory.
//   * Tiles are fetched in boxes of PG rows, the largest of 64, 32 or 16 that divides the page.  What lies behind a sequence's end in its last
//     page may be anything, NaN codes included: scores are selected by position, V rows are zeros there (CutMaps).
//   * The softmax warps read the query rows, cut them and write the swizzled operand themselves, at a piece's start.
//   * Issuers and producer run converged (tc_common.cuh).
#pragma once
#include "append_rope.cuh"  // pow2_scale, bf16_finite_max
#include "common.cuh"
#include "sched.cuh"
#include "tc_common.cuh"
#include "tc_decode_gqa_fp8_t.cuh"  // E4M3 descriptors and MMAs, tables in shared memory

namespace gqla {
namespace tc {

struct Fp8PagedParams {
    int32_t B, S, s_q, h_q, g, hpg;
    int32_t hb, hshift;      // heads of a row block (a power of two) and its logarithm: row r is position r >> hshift, head r & (hb - 1)
    int32_t n_hb, row_blocks;  // row blocks over the heads; over heads and positions
    int32_t balanced, W;
    int32_t plan_W, slack;   // of WholeOrBalanced
    int32_t n_rows, n_pages;
    float scale_log2;
    const __nv_bfloat16* q;  // [B, s_q, h_q, 576 or 192]
    const uint8_t* cache;    // absorb path: the latent rows, for prefetches into L2
    int32_t l2_stride;       // and the bytes between them; 0: none
    const float *k_scale, *r_scale, *v_scale;  // absorb path: k_scale [pages]; GQA path: [pages, g], [pages], [pages, g]
    RowMap rows;
    const int32_t* seqlens;
    float* o_part;    // [B, S, s_q, h_q, 512 or 128]
    float* lse_part;  // [B, S, s_q, h_q]
    int32_t* status;
};

template <int R, bool LATENT>
struct Fp8PagedSmem {
    static constexpr int kBlocks = LATENT ? 4 : 1;           // 128-column blocks of the keys in front of the RoPE part
    // Query rows: per 128-column block, and behind these for the RoPE part, 2 R rows of 128 (64) bytes, both terms' -- row r's hi term
    // in row qrow(r, 0), its lo term in qrow(r, 1).  Absorb path: runs of eight, hi and lo in turn, that multiply into 2 R
    // columns at once; GQA path: one term behind the other, multiplied into the same R columns.
    static constexpr bool kTermsApart = LATENT;
    __device__ static int qrow(int r, int term) { return kTermsApart ? (r >> 3) * 16 + term * 8 + (r & 7) : term * R + r; }
    static constexpr int kQBlock = 2 * R * 128;
    static constexpr int kQBytes = kBlocks * kQBlock + 2 * R * 64;
    static constexpr int kTokBytes = 16384;                  // 128 tokens x 128 bytes
    static constexpr int kKBytes = kBlocks * kTokBytes + 8192;
    static constexpr int kVBytes = LATENT ? 0 : kTokBytes;
    static constexpr int kStageBytes = kKBytes + kVBytes;
    static constexpr int kStages = LATENT ? 3 : 4;           // tiles on their way or in use (absorb path: of which some blocks only)
    // Absorb path: a ring of column blocks (128 tokens x 128 bytes), which P V frees one by one, and one of RoPE blocks, which Q K^T
    // frees.  Two and a quarter (R = 32) tiles fit; in two stages of a whole tile 64 x 4096 rows took 131 us, 128 heads.
    static constexpr int kColSlots = LATENT ? (R == 32 ? 9 : 10) : 0;
    static constexpr int kRingBytes = LATENT ? kColSlots * kTokBytes + kStages * 8192 : kStages * kStageBytes;
    static constexpr int kPRow = 2 * R;                      // one token's hi and lo terms, in runs of eight rows each
    static constexpr int kPBuf = 128 * kPRow;
    static constexpr int kOffStage = kQBytes;
    static constexpr int kOffRope = kOffStage + kColSlots * kTokBytes;  // (absorb path)
    static constexpr int kOffP = kOffStage + kRingBytes;
    static constexpr int kSoftmaxWarps = R / 2;              // R / 8 per TMEM lane quadrant, eight query rows a thread
    static constexpr int kOffRed = kOffP + 2 * kPBuf;        // [4][R] maxima, [R][4] sums, [R] factors of a raise, [R] references; the plan scratch
    static constexpr int kRedBytes = 2048;
    static constexpr int kOffScale = kOffRed + kRedBytes;    // [R] score scales of the piece's query rows
    // Scales of the tiles that the producer is ahead by, per run of a page: {K_C or latent, k_R, log2 V, 1 / V}.  The producer
    // is at most kStages + 1 tiles ahead of the one whose scores are looked at.
    static constexpr int kScaleTiles = 8;
    static constexpr int kOffPageScale = kOffScale + 128;
    static constexpr int kTileBytes = kOffPageScale + kScaleTiles * 8 * 16;
    // q_full o_free p_ready[2] pv_done[2] s_full[2] s_empty[2] kfull[] kempty[], GQA path: vfull[] vempty[], absorb path: cempty[]
    static constexpr int kNumBars = 10 + 2 * kStages + (LATENT ? kColSlots : 2 * kStages);
    static constexpr int kFirstSoftmax = 4;                  // warps 0, 1, 2: loads, Q K^T, P V
    static constexpr int kThreads = 32 * (kFirstSoftmax + kSoftmaxWarps);
    static constexpr int kTotal = kTileBytes + kNumBars * 8 + 16;
    static_assert(R == 16 || R == 32, "");
    static_assert(kScaleTiles >= kStages + 2 && R * 4 <= 128, "");
    static_assert(kQBytes % 1024 == 0 && kStageBytes % 1024 == 0 && kPBuf % 1024 == 0, "swizzled tiles need 1 KB alignment");
    static_assert(kRedBytes >= 10 * R * 4 && kRedBytes >= (3 * 32 + 4) * 4, "");
    static_assert(kTotal <= 232448, "shared memory budget of one CTA");
    static_assert(OneCtaPerSM<kTotal>::value, "");
};

constexpr float kP8Bias = 6.0f;   // log2 units a raised reference sits below the maximum that raised it
constexpr float kP8Grow = 8.75f;  // a score this far above its reference raises it: 2^8.75 = 430 < 448
constexpr float kP8Lo = 16.0f;    // scale of the second term

// Two values as two codes each: hi (nearest), lo (nearest to the rest, times kP8Lo).  By way of fp16, whose eleven bits add 2^-12
// to the 2^-9.
__device__ __forceinline__ void split_e4m3x2(float x0, float x1, uint16_t& hi, uint16_t& lo) {
    asm("{\n\t.reg .b32 h, b;\n\t"
        "cvt.rn.f16x2.f32 h, %3, %2;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 %0, h;\n\t"
        "cvt.rn.f16x2.e4m3x2 b, %0;\n\t"
        "sub.rn.f16x2 b, h, b;\n\t"
        "mul.rn.f16x2 b, b, %4;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 %1, b;\n\t}"
        : "=&h"(hi), "=h"(lo)
        : "f"(x0), "f"(x1), "r"(0x4c004c00u));  // 16, 16
}
__device__ __forceinline__ void split_e4m3x4(const float* x, uint32_t& hi, uint32_t& lo) {
    uint16_t h0, h1, l0, l1;
    split_e4m3x2(x[0], x[1], h0, l0);
    split_e4m3x2(x[2], x[3], h1, l1);
    hi = (uint32_t)h0 | ((uint32_t)h1 << 16);
    lo = (uint32_t)l0 | ((uint32_t)l1 << 16);
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// Asks for `bytes` (a multiple of 16) to be brought into L2.
__device__ __forceinline__ void prefetch_l2(const uint8_t* at, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(at), "r"(bytes) : "memory");
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Eight bf16 query elements times `inv` (a power of two: at most 448) as two codes each, hi (nearest) and lo (nearest to the rest).  By
// way of fp16, which holds the eight bits of what is not below 2^-14.  Codes have no infinity: of an infinite element the rest gets 0 x
// added, a NaN, as all scores of the row are then.
__device__ __forceinline__ void split_query8(const uint4& u, float inv, uint2& hi, uint2& lo) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint16_t h[4], l[4];
    const uint64_t inv2 = pack2(inv, inv);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x0, x1;
        unpack2(mul2(pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), inv2), x0, x1);
        asm("{\n\t.reg .b32 h, b;\n\t"
            "cvt.rn.f16x2.f32 h, %3, %2;\n\t"
            "cvt.rn.satfinite.e4m3x2.f16x2 %0, h;\n\t"
            "cvt.rn.f16x2.e4m3x2 b, %0;\n\t"
            "sub.rn.f16x2 b, h, b;\n\t"
            "fma.rn.f16x2 b, h, %4, b;\n\t"
            "cvt.rn.satfinite.e4m3x2.f16x2 %1, b;\n\t}"
            : "=&h"(h[i]), "=h"(l[i])
            : "f"(x0), "f"(x1), "r"(0u));
    }
    hi = make_uint2((uint32_t)h[0] | ((uint32_t)h[1] << 16), (uint32_t)h[2] | ((uint32_t)h[3] << 16));
    lo = make_uint2((uint32_t)l[0] | ((uint32_t)l[1] << 16), (uint32_t)l[2] | ((uint32_t)l[3] << 16));
}
// Two query rows of W bf16 elements in a warp, sixteen lanes each: fetched, scaled by a power of two and cut into two terms.
template <int W>
struct QueryPair {
    static constexpr int kChunks = W / 8, kPer = (kChunks + 15) / 16;
    uint4 u[kPer];
    __device__ __forceinline__ void fetch(const __nv_bfloat16* row, bool valid, int lane) {
#pragma unroll
        for (int c = 0; c < kPer; ++c) {
            const int ci = lane % 16 + 16 * c;
            u[c] = valid && ci < kChunks ? reinterpret_cast<const uint4*>(row)[ci] : make_uint4(0, 0, 0, 0);
        }
    }
    // Hands column 8 ci .. + 7's codes to store(first column, hi, lo); returns the row's scale.  sign: of the stored values.
    template <typename F>
    __device__ __forceinline__ float cut(int lane, float sign, F store) const {
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < kPer; ++c) top = bf16_max(top, u[c]);
        float amax = bf16_finite_max(top, [&](auto f) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) f(u[c]);
        });
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const float qs = amax > 0.f ? pow2_scale(amax, -110) : 1.f;
        const float inv = copysignf(__uint_as_float((254u << 23) - __float_as_uint(qs)), sign);  // 1 / qs
#pragma unroll
        for (int c = 0; c < kPer; ++c) {
            const int ci = lane % 16 + 16 * c;
            uint2 hi, lo;
            split_query8(u[c], inv, hi, lo);
            if (ci < kChunks) store(ci * 8, hi, lo);
        }
        return qs;
    }
};
// OR of a predicate over the `nthreads` threads that call it on named barrier `id`.  (Warps that meet in barriers leave a loop by
// such a vote, tc_common.cuh.)
__device__ __forceinline__ bool vote_any(int id, bool v, int nthreads) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(id), "r"((uint32_t)v), "r"(nthreads)
        : "memory");
    return r != 0;
}

template <int R, bool LATENT, int PG>
__global__ void __launch_bounds__(Fp8PagedSmem<R, LATENT>::kThreads, 1)
decode_fp8_paged_kernel(const Fp8PagedParams p, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmR,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CutMaps<PG> cut_maps) {
    using L = Fp8PagedSmem<R, LATENT>;
    constexpr int NS = L::kStages, NB = 128 / PG;
    constexpr int KB = L::kBlocks;
    constexpr int kQWidth = KB * 128 + 64;
    constexpr int kDv = KB * 128;  // value columns
    constexpr int kSmT = 32 * L::kSoftmaxWarps;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* tiles = smem_raw;
    if ((smem_u32(tiles) & 1023u) != 0) {  // swizzled tiles need 1 KB alignment
        if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, kStatusTimeout | (15 << 8));
        return;
    }
    uint8_t* q_smem = tiles;
    uint8_t* stage0 = tiles + L::kOffStage;
    uint8_t* p_smem = tiles + L::kOffP;
    float* red = reinterpret_cast<float*>(tiles + L::kOffRed);
    float* sums = red + 4 * R;
    float* factors = sums + 4 * R;
    float* refs = factors + R;
    float* sm_scale = reinterpret_cast<float*>(tiles + L::kOffScale);
    float4* page_scales = reinterpret_cast<float4*>(tiles + L::kOffPageScale);  // [tile % kScaleTiles][run]
    uint64_t* bars = reinterpret_cast<uint64_t*>(tiles + L::kTileBytes);
    uint64_t* q_full = bars + 0;
    uint64_t* o_free = bars + 1;
    uint64_t* p_ready = bars + 2;     // [2]
    uint64_t* pv_done = bars + 4;     // [2]
    uint64_t* s_full = bars + 6;      // [2]
    uint64_t* s_empty = bars + 8;     // [2]
    uint64_t* kfull = bars + 10;       // the tile's keys (absorb path: all of it)
    uint64_t* kempty = kfull + NS;    // Q K^T has read them (absorb path: the RoPE part may go)
    uint64_t* vfull = kempty + NS;    // GQA path
    uint64_t* vempty = vfull + NS;
    uint64_t* cempty = kempty + NS;   // absorb path: [kColSlots], P V has read the column block
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::kNumBars);
    volatile int32_t* abort_flag = reinterpret_cast<volatile int32_t*>(tmem_slot + 1);

    // TMEM columns: the score buffers (absorb path: the products with the two terms apart; GQA path: the K_C and the k_R products apart,
    // they have scales of their own), then O^T, one block of 2 R columns per 128 value columns: row r's hi products in column
    // 16 (r / 8) + r % 8, its lo products eight further on
    constexpr int kScols = 2 * R;
    constexpr uint32_t kColS = 0, kColO = 2 * kScols, kColsUsed = kColO + KB * 2 * R;
    constexpr uint32_t kTmemCols = kColsUsed <= 128 ? 128 : (kColsUsed <= 256 ? 256 : 512);

    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const Abort ab{abort_flag, p.status};

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kNumBars; ++i) {
            const bool per_warp = i < 4 || (&bars[i] >= s_empty && &bars[i] < kfull);  // q_full, o_free, p_ready, s_empty
            mbar_init(&bars[i], per_warp ? L::kSoftmaxWarps : 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, kTmemCols);
        tmem_relinquish();
    }
    pdl_launch_dependents();
    if (warp == 0 && elect_one()) {
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmR);
        if (!LATENT) tma_prefetch_desc(&tmV);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);
    pdl_wait();  // set-up is done (behind the preceding kernel's tail); everything below reads the caller's tensors
    const int rb = blockIdx.x % p.row_blocks;
    const int j = blockIdx.x / p.row_blocks % p.g;
    const int unit = blockIdx.x / (p.row_blocks * p.g);
    const int i0 = rb % p.n_hb * p.hb;                  // first head of this row block in its group
    const int pq0 = rb / p.n_hb * (R >> p.hshift);      // first query position
    WholeOrBalanced walk;
    if (p.balanced) {
        walk.init_balanced(p.seqlens, p.B, p.S, unit, p.W, p.plan_W, p.slack, reinterpret_cast<int32_t*>(red), L::kThreads);
    } else {
        walk.init_fixed(p.seqlens, p.B, p.S, unit / p.S, unit % p.S);
    }
    Piece pc;
    int gt = 0;  // tiles walked so far: S / P buffer = gt & 1, phase = (gt >> 1) & 1
    int pi = 0;  // non-empty pieces walked so far

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        const uint32_t e = elect_one();
        const uint32_t page_step = 128u / (uint32_t)p.rows.page_size, page_rest = 128u % (uint32_t)p.rows.page_size;
        int s = 0, cs = 0;  // next slots: of tiles, of column blocks
        int pt = 0;         // tiles loaded so far
        uint32_t ph = 1, cph = 1;  // parity that means "slot is free"
        bool ok = true;
        while (ok && warp_all(walk.next(pc))) {
            const int n_tiles = warp_uniform(pc.n_tiles);
            if (n_tiles == 0) continue;
            const int32_t T = p.seqlens[pc.b];
            // the query rows, which the softmax warps read when they are through with the piece before: the heads of a position are together
            if (lane < (R >> p.hshift) && pq0 + lane < p.s_q)
                prefetch_l2(reinterpret_cast<const uint8_t*>(p.q + (((int64_t)pc.b * p.s_q + pq0 + lane) * p.h_q + (int64_t)j * p.hpg + i0) * kQWidth),
                            (uint32_t)((p.hpg - i0 < p.hb ? p.hpg - i0 : p.hb) * kQWidth * 2));
            // This lane's run of the tile that is looked up next: its first token, that one's place in its page, the page's in the
            // block table.  Page numbers are looked up two tiles ahead, scales one.
            const int run = lane % NB;
            const int32_t* table = p.rows.block_table + (int64_t)pc.b * p.rows.max_pages;
            uint32_t tok = (uint32_t)(pc.tok_begin + run * PG);
            uint32_t col = tok / (uint32_t)p.rows.page_size, at = tok - col * p.rows.page_size;
            auto next_run = [&](int32_t& page, uint32_t& in_page) {
                page = tok < (uint32_t)T && col < (uint32_t)p.rows.max_pages ? table[col] : -1;  // (the block table says nothing about pages behind the end)
                in_page = at;
                tok += 128u;
                col += page_step;
                at += page_rest;
                if (at >= (uint32_t)p.rows.page_size) {
                    at -= p.rows.page_size;
                    ++col;
                }
            };
            struct Scales { float k, r, v; };
            auto scales_of = [&](int32_t page) -> Scales {
                if ((uint32_t)page >= (uint32_t)p.n_pages) return {1.f, 1.f, 1.f};
                if (LATENT) {
                    const float s = p.k_scale[page];
                    return {s, s, s};
                }
                return {p.k_scale[(int64_t)page * p.g + j], p.r_scale[page], p.v_scale[(int64_t)page * p.g + j]};
            };
            int32_t page, page1, page2;
            uint32_t in_page, in_page1, in_page2;
            next_run(page, in_page);
            next_run(page1, in_page1);
            Scales cur = scales_of(page);
            for (int t = 0; t < n_tiles; ++t, ++pt) {
                const int32_t row = page < 0 ? p.n_rows : (int32_t)((int64_t)page * p.rows.page_size + in_page);
                const int32_t left = T - (pc.tok_begin + t * 128);
                const int cut = (int)warp_uniform((uint32_t)cut_run<PG>(left, 128));
                next_run(page2, in_page2);
                const Scales next = scales_of(page1);
                // (a row block each of the tile after next: its rows are in L2 when a slot is free for them)
                if (LATENT && p.l2_stride > 0 && lane < NB && t + 1 < pc.n_tiles && (t + 1) % p.row_blocks == rb && (uint32_t)page1 < (uint32_t)p.n_pages) {
                    const int32_t rows_left = left - 128 - run * PG;
                    const int32_t n = rows_left < PG ? rows_left : PG;
                    if (n > 0)
                        prefetch_l2(p.cache + ((int64_t)page1 * p.rows.page_size + in_page1) * p.l2_stride, (uint32_t)((n - 1) * p.l2_stride + 576));
                }
                int32_t y[NB];  // first cache row of each run
#pragma unroll
                for (int rn = 0; rn < NB; ++rn) y[rn] = __shfl_sync(0xffffffffu, row, rn);
                const int32_t y_cut = __shfl_sync(0xffffffffu, row, cut < 0 ? 0 : cut);
                // The tile's scales are published with its first barrier: whoever sees its scores sees them.
                auto publish_scales = [&]() {
                    if (lane < NB) {  // (the logarithm of a scale of zero would not be finite)
                        const float sv = fmaxf(cur.v, 8.6736174e-19f);
                        page_scales[pt % L::kScaleTiles * 8 + lane] = make_float4(cur.k, cur.r, lg2(sv), rcp(sv));
                    }
                    __syncwarp();
                };
                if constexpr (LATENT) {
                    if (!(ok = warp_all(mbar_wait(&kempty[s], ph, ab, 1)))) break;
                    publish_scales();
                    mbar_expect_tx(&kfull[s], L::kKBytes, e);
                    __syncwarp();
                    uint8_t* rope_dst = tiles + L::kOffRope + s * 8192;
#pragma unroll
                    for (int rn = 0; rn < NB; ++rn) tma_load_2d(rope_dst + rn * PG * 64, &tmR, 512, y[rn], &kfull[s], e);
#pragma unroll 1
                    for (int m = 0; m < KB; ++m) {
                        uint8_t* dst = stage0 + cs * L::kTokBytes;
                        if (!(ok = warp_all(mbar_wait(&cempty[cs], cph, ab, 2)))) break;
#pragma unroll
                        for (int rn = 0; rn < NB; ++rn)
                            tma_load_2d(dst + rn * PG * 128, &tmK, m * 128, y[rn], &kfull[s], rn != cut ? e : 0u);
                        if (cut >= 0)
                            load_cut_run<PG, 1>(cut_maps, lane, left % PG, y_cut, p.n_rows, [&](const CUtensorMap* map, int, int r, int32_t yy) {
                                tma_load_2d(dst + cut * PG * 128 + r * 128, map, m * 128, yy, &kfull[s]);
                            });
                        if (++cs == L::kColSlots) { cs = 0; cph ^= 1; }
                    }
                    if (!ok) break;
                } else {
                    uint8_t* st = stage0 + s * L::kStageBytes;
                    uint8_t* sv = st + L::kKBytes;
                    if (!(ok = warp_all(mbar_wait(&kempty[s], ph, ab, 1)))) break;
                    publish_scales();
                    mbar_expect_tx(&kfull[s], L::kKBytes, e);
                    __syncwarp();
#pragma unroll
                    for (int rn = 0; rn < NB; ++rn) tma_load_3d(st + rn * PG * 128, &tmK, 0, j, y[rn], &kfull[s], e);
#pragma unroll
                    for (int rn = 0; rn < NB; ++rn) tma_load_2d(st + L::kTokBytes + rn * PG * 64, &tmR, 0, y[rn], &kfull[s], e);
                    if (!(ok = warp_all(mbar_wait(&vempty[s], ph, ab, 2)))) break;
                    mbar_expect_tx(&vfull[s], L::kVBytes, e);
                    __syncwarp();
#pragma unroll
                    for (int rn = 0; rn < NB; ++rn) tma_load_3d(sv + rn * PG * 128, &tmV, 0, j, y[rn], &vfull[s], rn != cut ? e : 0u);
                    if (cut >= 0)
                        load_cut_run<PG, 1>(cut_maps, lane, left % PG, y_cut, p.n_rows, [&](const CUtensorMap* map, int, int r, int32_t yy) {
                            tma_load_3d(sv + cut * PG * 128 + r * 128, map, 0, j, yy, &vfull[s]);
                        });
                }
                if (++s == NS) { s = 0; ph ^= 1; }
                page = page1; in_page = in_page1;
                page1 = page2; in_page1 = in_page2;
                cur = next;
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer of Q K^T
        // (Q K^T and P V have a warp each, so that neither waits for what the other needs: absorb path, 64 x 4096 rows, 128 heads 116
        // us; both in one warp 134)
        const uint32_t e = elect_one();
        constexpr uint32_t idesc = idesc_e4m3(128, L::kTermsApart ? 2 * R : R, 0, 0);  // S^T: A = K tile (K-major), B = Q (K-major)
        constexpr int kTerms = L::kTermsApart ? 1 : 2;                                 // passes over the keys
        const uint32_t q_lo = desc_lo(desc_kmajor_sw128(smem_u32(q_smem)));
        const uint32_t qr_lo = desc_lo(desc_kmajor_sw64(smem_u32(q_smem + KB * L::kQBlock)));
        int s = 0, cs = 0;
        uint32_t ph = 0;
        bool ok = true;
        while (ok && warp_all(walk.next(pc))) {
            const int n_tiles = warp_uniform(pc.n_tiles);
            if (n_tiles == 0) continue;
            if (!(ok = warp_all(mbar_wait(q_full, pi & 1, ab, 4)))) break;
            for (int t = 0; t < n_tiles; ++t) {
                const int n = gt + t;
                if (!(ok = warp_all(mbar_wait_fast(&s_empty[n & 1], ((n >> 1) & 1) ^ 1, ab, 10)))) break;
                if (!(ok = warp_all(mbar_wait_fast(&kfull[s], ph, ab, 3)))) break;
                tc_fence_after();
                const uint32_t d = tmem_base + kColS + (uint32_t)(n & 1) * kScols;
                const uint8_t* rope = LATENT ? tiles + L::kOffRope + s * 8192 : stage0 + s * L::kStageBytes + L::kTokBytes;
                const uint32_t r_lo = desc_lo(desc_kmajor_sw64(smem_u32(rope)));
#pragma unroll
                for (int m = 0; m < KB; ++m) {
                    const uint32_t k_lo = desc_lo(desc_kmajor_sw128(smem_u32(stage0 + (LATENT ? cs * L::kTokBytes : s * L::kStageBytes))));
#pragma unroll
                    for (int term = 0; term < kTerms; ++term)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)  // 32 elements a step
                            umma_f8_ss_lo(d, k_lo + ((kk * 32) >> 4), kDescHiSw128,
                                          q_lo + ((m * L::kQBlock + term * R * 128 + kk * 32) >> 4), kDescHiSw128, idesc, (m | term | kk) != 0, e);
                    if (LATENT && ++cs == L::kColSlots) cs = 0;
                }
#pragma unroll
                for (int term = 0; term < kTerms; ++term)
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk)
                        umma_f8_ss_lo(LATENT ? d : d + R, r_lo + ((kk * 32) >> 4), kDescHiSw64, qr_lo + ((term * R * 64 + kk * 32) >> 4),
                                      kDescHiSw64, idesc, LATENT || (term | kk) != 0, e);
                umma_commit(&s_full[n & 1], e);
                umma_commit(&kempty[s], e);
                if (++s == NS) { s = 0; ph ^= 1; }
            }
            gt += n_tiles;
            ++pi;
        }
    } else if (warp == 2) {
        // ------------------------------------------------------------------ MMA issuer of P V
        const uint32_t e = elect_one();
        constexpr uint32_t idesc = idesc_e4m3(128, 2 * R, 1, 1);  // O^T: A = V tile read MN-major, B = P^T rows (MN-major)
        const uint64_t pd0 = desc_mnmajor_rows(smem_u32(p_smem), L::kPRow);
        int s = 0;  // column block (absorb path) or tile
        uint32_t ph = 0;
        bool ok = true;
        while (ok && warp_all(walk.next(pc))) {
            const int n_tiles = warp_uniform(pc.n_tiles);
            if (n_tiles == 0) continue;
            for (int t = 0; t < n_tiles; ++t) {
                const int n = gt + t;
                if (!(ok = warp_all(mbar_wait_fast(&p_ready[n & 1], (n >> 1) & 1, ab, 5)))) break;
                if (t == 0 && pi > 0 && !(ok = warp_all(mbar_wait(o_free, (pi - 1) & 1, ab, 14)))) break;
                if (!LATENT && !(ok = warp_all(mbar_wait_fast(&vfull[s], ph, ab, 6)))) break;
                tc_fence_after();
                const uint32_t p_lo = (uint32_t)pd0 + (((n & 1) * L::kPBuf) >> 4);
#pragma unroll
                for (int m = 0; m < KB; ++m) {
                    const uint64_t vd = desc_mnmajor_sw128(smem_u32(stage0 + (LATENT ? s * L::kTokBytes : s * L::kStageBytes + L::kKBytes)), 16384);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // 32 tokens a step
                        umma_f8_ss_lo(tmem_base + kColO + (uint32_t)m * 2 * R, (uint32_t)vd + ((kk * 4096) >> 4), (uint32_t)(vd >> 32),
                                      p_lo + ((kk * 32 * L::kPRow) >> 4), (uint32_t)(pd0 >> 32), idesc, (t | kk) != 0, e);
                    umma_commit(LATENT ? &cempty[s] : &vempty[s], e);
                    if (++s == (LATENT ? L::kColSlots : NS)) { s = 0; ph ^= 1; }
                }
                umma_commit(&pv_done[n & 1], e);
            }
            gt += n_tiles;
            ++pi;
        }
    } else if (warp >= L::kFirstSoftmax) {
        // ------------------------------------------------------------------ softmax: one TMEM lane = one token per thread
        const int q = warp & 3;
        const int sw = warp - L::kFirstSoftmax;
        const int part = sw >> 2;            // which eight of the query rows
        const int r0 = part * 8;
        const int bar = 2 + part;            // barrier of the four warps that have these rows
        const int tl = q * 32 + lane;        // token within the tile == TMEM lane (and value column in the output)
        const uint32_t lane_base = tmem_base + ((uint32_t)(q * 32) << 16);
        const int sq_left = p.s_q - pq0;  // query positions of this block and behind it
        // rows [0, r_hi) stand for positions of the step (those of heads behind the group's are computed and dropped)
        const int r_hi = sq_left < (R >> p.hshift) ? sq_left << p.hshift : R;
        const int hmask = p.hb - 1;
        // this thread's sixteen bytes of its token's row of P^T: the hi terms of its eight rows, then the lo terms
        uint8_t* prow = p_smem + tl * L::kPRow + (((uint32_t)part ^ (((uint32_t)(tl * L::kPRow) >> 7) & (R == 32 ? 3u : 1u))) << 4);
        float m_ref[8], l[8];

        while (walk.next(pc)) {
            const int32_t T = p.seqlens[pc.b];
            const int64_t slot0 = (int64_t)pc.b * p.S;
            GQLA_DEBUG_CHECK(pc.b >= 0 && pc.b < p.B, p.status, 32);
            GQLA_DEBUG_CHECK(pc.n_tiles == 0 || (pc.k >= 0 && pc.k < p.S), p.status, 33);
            GQLA_DEBUG_CHECK(pc.tok_begin >= 0 && pc.tok_begin <= pc.tok_end && pc.tok_end <= (T > 0 ? T : 0), p.status, 34);
            if (part == 0 && tl < R) {  // split slots this worker marks empty (thread r speaks for row r)
                const int pq = pq0 + (tl >> p.hshift), il = i0 + (tl & hmask);
                if (il < p.hpg && pq < p.s_q)
                    for (int kk = pc.fill_begin; kk < pc.fill_end; ++kk)
                        p.lse_part[((slot0 + kk) * p.s_q + pq) * p.h_q + (int64_t)j * p.hpg + il] = -INFINITY;
            }
            if (pc.n_tiles == 0 && p.balanced) continue;
            if (pc.n_tiles > 0) {
                // ---------------------------------------------------------- the piece's query rows, two a warp
                // (the scores of the previous piece's last tile have been read, so nothing reads the old rows any more)
                const int r = 2 * sw + (lane >> 4), pq = pq0 + (r >> p.hshift), il = i0 + (r & hmask);
                QueryPair<kQWidth> rows;
                rows.fetch(p.q + (((int64_t)pc.b * p.s_q + pq) * p.h_q + (int64_t)j * p.hpg + il) * kQWidth, il < p.hpg && pq < p.s_q, lane);
                const float qs = rows.cut(lane, 1.f, [&](int col, const uint2& hi, const uint2& lo) {
                    // blocks of 128 columns: 128-byte rows, 16-byte chunks XORed with r % 8; the RoPE block: 64-byte rows, with r / 2 % 4
                    const int blk = col / 128, pitch = blk < KB ? 128 : 64;
                    uint8_t* at = q_smem + (blk < KB ? blk * L::kQBlock + ((((col % 128) >> 4) ^ (r & 7)) << 4)
                                                     : KB * L::kQBlock + ((((col - KB * 128) >> 4) ^ ((r >> 1) & 3)) << 4)) + (col & 8);
                    *reinterpret_cast<uint2*>(at + L::qrow(r, 0) * pitch) = hi;
                    *reinterpret_cast<uint2*>(at + L::qrow(r, 1) * pitch) = lo;
                });
                if (lane % 16 == 0) sm_scale[r] = p.scale_log2 * qs;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
            }
            named_bar_sync(1, kSmT);  // the scales are there
#pragma unroll
            for (int r = 0; r < 8; ++r) m_ref[r] = l[r] = 0.f;  // (a row that sees a token of the piece sees one of its first tile)
            bool ok = true;
            // tokens below this are visible to every row of a block without positions behind the step's
            const int all_end = r_hi < R ? INT32_MIN : (T - (sq_left - 1) < pc.tok_end ? T - (sq_left - 1) : pc.tok_end);

            for (int t = 0; t < pc.n_tiles && ok; ++t) {
                const int n = gt + t;
                const int s = n & 1;
                // A wait that fails raises the CTA's abort flag; the warps agree on leaving at the next barrier below
                // (a warp that left the loop on its own would strand the others in that barrier).
                bool okl = __all_sync(0xffffffffu, mbar_wait_fast(&s_full[s], (n >> 1) & 1, ab, 7));
                tc_fence_after();
                float d[8], inv_sv;  // scores above their references, log2 units
                {
                    uint32_t x[16];  // absorb path: the hi and the lo terms' products of rows r0 .. r0 + 7; GQA path: K_C's and k_R's
                    if (okl) {
                        const uint32_t at = lane_base + kColS + (uint32_t)s * kScols;
                        if (LATENT) {
                            tmem_ld16(at + 2 * r0, x);
                        } else {
                            tmem_ld8(at + r0, x);
                            tmem_ld8(at + R + r0, x + 8);
                        }
                        tmem_wait_ld();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && okl) mbar_arrive(&s_empty[s]);  // the scores have been read
                    float rs[8];
                    load_row<8>(rs, sm_scale + r0);
                    const float4 ps = page_scales[n % L::kScaleTiles * 8 + tl / PG];
                    const uint64_t s0 = pack2(ps.x, ps.x), s1 = pack2(ps.y, ps.y), up = pack2(ps.z, ps.z), minus = pack2(-1.f, -1.f);
#pragma unroll
                    for (int c = 0; c < 8; c += 2) {
                        const uint64_t x0 = pack2(__uint_as_float(x[c]), __uint_as_float(x[c + 1]));
                        const uint64_t x1 = pack2(__uint_as_float(x[c + 8]), __uint_as_float(x[c + 9]));
                        const uint64_t dot = LATENT ? mul2(add2(x0, x1), s0) : fma2(x0, s0, mul2(x1, s1));
                        unpack2(fma2(dot, pack2(rs[c], rs[c + 1]), fma2(pack2(m_ref[c], m_ref[c + 1]), minus, up)), d[c], d[c + 1]);
                    }
                    inv_sv = ps.w;
                }
                if (!okl || pc.tok_begin + (t + 1) * 128 > all_end) {
                    // rows this thread's token is visible to: the token at absolute position ta is seen by query positions
                    // pq >= s_q - (T - ta); positions behind the step's see nothing
                    const int ta = pc.tok_begin + t * 128 + tl;
                    const int pq_min = sq_left - (T - ta) > 0 ? sq_left - (T - ta) : 0;  // counted from this block's first
                    const int r_lo = okl && ta < pc.tok_end && pq_min < 32 ? (pq_min << p.hshift) : R;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (r0 + c < r_lo || r0 + c >= r_hi) d[c] = -INFINITY;
                }
                float top = d[0];
#pragma unroll
                for (int c = 1; c < 8; ++c) top = fmaxf(top, d[c]);
                if (t == 0 || vote_any(bar, top > kP8Grow || !okl, 128)) {  // a piece's first tile sets the references in any case
                    float* redw = red + q * R + r0;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float wm = warp_max_redux(d[c]);
                        if (lane == 0) redw[c] = wm;
                    }
                    if (vote_any(bar, !okl, 128)) { ok = false; break; }  // leaving is agreed on (tc_common.cuh)
                    float* factor = factors + r0;
                    bool any = false;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const int r = r0 + c;
                        const float up = fmaxf(fmaxf(red[r], red[R + r]), fmaxf(red[2 * R + r], red[3 * R + r]));
                        const bool need = up > (t == 0 ? -FLT_MAX : kP8Grow);
                        const float by = need ? up - kP8Bias : 0.f;
                        const float f = ex2(-by);  // (on the first tile there is nothing to scale yet)
                        any |= need;
                        l[c] *= f;
                        m_ref[c] += by;
                        d[c] -= by;
                        if (lane == 0) factor[c] = f;  // (the same from the four warps)
                    }
                    named_bar_sync(bar, 128);  // red may be rewritten by the next tile; the factors are there
                    if (any && t > 0) {  // the same in the four warps; no barrier follows inside this branch
                        // O^T may be rescaled only between P.V(n-1) completing and P.V(n) being issued
                        if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[(n - 1) & 1], ((n - 1) >> 1) & 1, ab, 8))) {
                            okl = false;  // noticed by everybody at the next barrier
                        } else {
                            tc_fence_after();
#pragma unroll 1
                            for (int m = 0; m < KB; ++m) {
                                uint32_t o[16];
                                tmem_ld16(lane_base + kColO + (uint32_t)m * 2 * R + 2 * r0, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * factor[c & 7]);
                                tmem_st16(lane_base + kColO + (uint32_t)m * 2 * R + 2 * r0, o);
                            }
                            tmem_wait_st();
                        }
                    }
                }
                // P^T buffer s was last read by P.V(n-2)
                if (okl && t > 1) okl = __all_sync(0xffffffffu, mbar_wait_fast(&pv_done[s], ((n - 2) >> 1) & 1, ab, 8));
                // weights of this token -> its sixteen bytes of P^T
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int c = 0; c < 8; c += 2) {
                    d[c] = ex2(d[c]);
                    d[c + 1] = ex2(d[c + 1]);
                    unpack2(fma2(pack2(d[c], d[c + 1]), pack2(inv_sv, inv_sv), pack2(l[c], l[c + 1])), l[c], l[c + 1]);
                }
                split_e4m3x4(d, hi[0], lo[0]);
                split_e4m3x4(d + 4, hi[1], lo[1]);
                *reinterpret_cast<uint4*>(prow + s * L::kPBuf) = make_uint4(hi[0], hi[1], lo[0], lo[1]);
                fence_proxy_async_smem();  // generic-proxy writes of P^T -> visible to the tensor core
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && okl) mbar_arrive(&p_ready[s]);
            }

            // -------------------------------------------------------------- row sums across the 128 tokens, then the output
            // (the sums do not need the last P.V, so they are exchanged while it runs)
            warp_sums_scatter<8>(l, lane);
            if (lane % 4 == 0) sums[4 * (r0 + lane / 4) + q] = l[0];
            if (q == 0 && lane == 0) store_row<8>(refs + r0, m_ref);
            const int n_last = gt + pc.n_tiles - 1;
            if (pc.n_tiles > 0 && ok)
                ok = __all_sync(0xffffffffu, mbar_wait_fast(&pv_done[n_last & 1], (n_last >> 1) & 1, ab, 9));
            tc_fence_after();
            named_bar_sync(1, kSmT);
            const int64_t out_row0 = ((slot0 + pc.k) * p.s_q) * p.h_q + (int64_t)j * p.hpg;
            // lane c finishes row c of the eight, the others get its factor
            float f;
            {
                const int r = r0 + lane % 8, pq = pq0 + (r >> p.hshift), il = i0 + (r & hmask);
                const float4 s4 = *reinterpret_cast<const float4*>(sums + 4 * r);
                const float Lt = ok && pc.n_tiles > 0 ? (s4.x + s4.y) + (s4.z + s4.w) : 0.f;
                f = Lt == 0.f ? 0.f : 1.f / Lt;  // zero: the row sees nothing (its largest weight is at least 2^6 otherwise, or NaN)
                if (q == 0 && lane < 8 && il < p.hpg && pq < p.s_q)
                    p.lse_part[out_row0 + (int64_t)pq * p.h_q + il] = Lt == 0.f ? -INFINITY : (refs[r] + log2f(Lt)) * 0.6931471805599453f;
            }
#pragma unroll 1
            for (int m = 0; m < KB; ++m) {
                float acc[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = 0.f;
                if (pc.n_tiles > 0 && ok) {  // warp-uniform
                    uint32_t o[2][8];        // hi and lo terms' products
                    tmem_ld8(lane_base + kColO + (uint32_t)m * 2 * R + 2 * r0, o[0]);
                    tmem_ld8(lane_base + kColO + (uint32_t)m * 2 * R + 2 * r0 + 8, o[1]);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float w = __shfl_sync(0xffffffffu, f, c);
                        if (w != 0.f) acc[c] = fmaf(__uint_as_float(o[1][c]), 1.f / kP8Lo, __uint_as_float(o[0][c])) * w;
                    }
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const int rc = r0 + c, pq = pq0 + (rc >> p.hshift), il = i0 + (rc & hmask);
                    // lane tl holds value column 128 m + tl of every row: 128 consecutive floats per row
                    if (il < p.hpg && pq < p.s_q) p.o_part[(out_row0 + (int64_t)pq * p.h_q + il) * kDv + m * 128 + tl] = acc[c];
                }
            }
            named_bar_sync(1, kSmT);  // the tables may be rewritten by the next piece
            // O^T has been read: the next piece's first P.V may overwrite it
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
            gt += pc.n_tiles;
            if (pc.n_tiles > 0) ++pi;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
}

}  // namespace tc
}  // namespace gqla
