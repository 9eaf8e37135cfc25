// Absorb-path split-KV flash decoding over E4M3 pages with a scale per page (Eq. (mqa), lines 3-5) with the QUERY ROWS on the MMA's M
// axis, for more than 64 of them and enough pieces: the CTA-pair design of tc_decode_absorb_fp8.cuh (2-CTA cluster, cta_group::2 MMAs of M = 128, each CTA
// 64 query rows, O in 256 TMEM columns, S in 64) with the precision and the page handling of tc_decode_fp8_paged.cuh.  That kernel
// takes 128 rows as four CTAs, which read every tile from L2 four times and keep it in shared memory for 32 rows' work;
// here a pair reads it once (K and V boxes), for 128.
//
// Bound by the tensor core and by a piece's ends: a tile's MMAs take about 2540 cycles back to back and a tile 2650
// to 2800 (tensor pipe active 56 % of the SM's cycles); a piece costs another 18000 (queries 6000, first references 5000, output 7000).  128 heads, 64 x 4096 rows:
// 76 us merge included in a graph of 18 passes, 0.96 PFLOP/s of the method's products, each done twice here; 90 to 92 at the power cap.
//
//   * Queries: hi and lo, both E4M3, written to shared memory by the softmax warps at a piece's start; S = (Q_hi + Q_lo) K^T in one
//     accumulator, 36 MMAs a tile.
//   * Weights P' = 2^(y - m), y = x + log2 s (the page's scale is the values' scale, too): hi is E4M3, lo the rest as E5M2 in the same
//     accumulator, whose smaller range would cost an E4M3 lo its bits -- three significant bits behind four leave 2^-8 of P', and E5M2
//     reaches 2^-16, i.e. 2^-22 of a row's largest weight (which is at least 2^6).
//   * A softmax thread has 32 tokens of one row, which are at most two pages: two scales a tile, looked up by the K producer
//     with the rows and passed through shared memory behind a barrier of their own (the tile's full barriers are the leader CTA's).
//   * Shared memory: two terms of Q 72 KB, of P 16 KB, K in a ring of three half tiles, V in one of four.
#pragma once
#include "append_rope.cuh"  // pow2_scale
#include "common.cuh"
#include "sched.cuh"
#include "tc_common.cuh"
#include "tc_decode_absorb_fp8.cuh"  // cta_group::2 MMAs of kind::f8f6f4, descriptors
#include "tc_decode_fp8_paged.cuh"   // scales' arithmetic

namespace gqla {
namespace tc {

struct Fp8PairParams {
    int32_t B, S, s_q, h_q, rows_total /* s_q*h_q */, row_blocks /* ceil(rows_total/128) */;
    int32_t balanced, W;  // balanced plan: W pairs per row block, grid = 2 * W * row_blocks
    int32_t slack;        // of WholeOrBalanced
    int32_t n_rows, n_pages;
    float scale_log2;
    const __nv_bfloat16* q;   // [B, s_q * h_q, 576]
    const float* page_scale;  // [pages]
    RowMap rows;
    const int32_t* seqlens;
    float* o_part;    // [B, S, s_q*h_q, 512]
    float* lse_part;  // [B, S, s_q*h_q]
    int32_t* status;
};

struct Fp8PairSmem {
    static constexpr int kBox = 8192;                 // 64 rows x 128 E4M3, 128-byte swizzle
    static constexpr int kRBox = 4096;                // 64 rows x 64 E4M3 (RoPE part), 64-byte swizzle
    static constexpr int kQTerm = 4 * kBox + kRBox;   // 64 query rows x 576, one term
    static constexpr int kPTerm = kBox;               // 64 rows x 128 tokens, one term
    static constexpr int kPBytes = 2 * kPTerm;
    static constexpr int kKGroup = 2 * kBox + kRBox;  // group 0: latent boxes 0, 1;  group 1: boxes 2, 3 and the RoPE box
    static constexpr int kVGroup = 2 * kBox;          // 64 tokens x this CTA's 2 x 128 latent columns
    static constexpr int kNK = 3;                     // ring of K groups: a tile and a half
    static constexpr int kNV = 4;                     // ring of V groups: two tiles
    static constexpr int kOffP = 2 * kQTerm;
    static constexpr int kOffV = kOffP + kPBytes;     // P and the V ring are contiguous: together the output staging
    static constexpr int kOffK = kOffV + kNV * kVGroup;
    static constexpr int kScaleTiles = 8;             // the K producer is at most three tiles ahead of the softmax
    static constexpr int kOffScale = kOffK + kNK * kKGroup;      // [kScaleTiles][8 runs of 16 tokens] {scale, log2, 1 / scale, -}
    static constexpr int kOffRow = kOffScale + kScaleTiles * 8 * 16;  // [64] score scales of the piece's query rows
    static constexpr int kOffMax = kOffRow + 64 * 4;  // [4][64] maxima of a raise, sums at a piece's end; the plan scratch
    static constexpr int kTileBytes = kOffMax + 2048;
    // kfull[kNK] kempty[kNK] vfull[kNV] vempty[kNV] q_full o_free epi_done s_full[2] p_ready[2] pv_done[2] fin sc_full[kScaleTiles]
    static constexpr int kNumBars = 2 * kNK + 2 * kNV + 10 + kScaleTiles;
    static constexpr int kSoftmaxWarps = 8;
    static constexpr int kVProducerWarp = 2 + kSoftmaxWarps;
    static constexpr int kThreads = 96 + 32 * kSoftmaxWarps;
    static constexpr int kWarpPitch = 64 * 4 + 16;    // fp32 partials: a softmax warp's 32 rows x 64 columns
    static_assert(8 * 32 * kWarpPitch <= kPBytes + kNV * kVGroup, "output staging must fit in P + V ring");
    static_assert(kQTerm % 1024 == 0 && kKGroup % 1024 == 0 && kOffP % 1024 == 0, "swizzled tiles need 1 KB alignment");
    static constexpr int kTotal = kTileBytes + kNumBars * 8 + 16;
    static_assert(2048 >= (kThreads + 4) * 4, "plan scratch must fit in the table of maxima");
    static_assert(kTotal <= 232448, "shared memory budget of one CTA");
    static_assert(OneCtaPerSM<kTotal>::value, "");
};

// Two values as two codes each: hi in E4M3 (nearest), lo in E5M2 (nearest to the rest).  By way of fp16, whose eleven bits add 2^-12.
__device__ __forceinline__ void split_e4m3_e5m2(float x0, float x1, uint16_t& hi, uint16_t& lo) {
    asm("{\n\t.reg .b32 h, b;\n\t"
        "cvt.rn.f16x2.f32 h, %3, %2;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 %0, h;\n\t"
        "cvt.rn.f16x2.e4m3x2 b, %0;\n\t"
        "sub.rn.f16x2 b, h, b;\n\t"
        "cvt.rn.satfinite.e5m2x2.f16x2 %1, b;\n\t}"
        : "=&h"(hi), "=h"(lo)
        : "f"(x0), "f"(x1));
}

// Page and place in it of a run of tokens, tile after tile.
struct PageWalk {
    const int32_t* table;
    uint32_t tok, col, at, page_size, step, rest, max_pages;
    int32_t T;
    __device__ __forceinline__ PageWalk(const RowMap& rows, int32_t b, uint32_t first, int32_t T_)
        : table(rows.block_table + (int64_t)b * rows.max_pages), tok(first), page_size(rows.page_size), step(128u / page_size),
          rest(128u % page_size), max_pages(rows.max_pages), T(T_) {
        col = tok / page_size;
        at = tok - col * page_size;
    }
    __device__ __forceinline__ void next(int32_t& page, uint32_t& in_page) {  // -1 behind the sequence's end
        page = tok < (uint32_t)T && col < max_pages ? table[col] : -1;
        in_page = at;
        tok += 128u;
        col += step;
        at += rest;
        if (at >= page_size) {
            at -= page_size;
            ++col;
        }
    }
};

template <int PG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Fp8PairSmem::kThreads, 1)
decode_fp8_pair_kernel(const Fp8PairParams p, const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmCr,
                       const __grid_constant__ CutMaps<PG> cut_maps) {
    using L = Fp8PairSmem;
    constexpr int NB = 64 / PG;  // boxes of a column block of half a tile
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* tiles = smem_raw;
    if ((smem_u32(tiles) & 1023u) != 0) {  // swizzled tiles need 1 KB alignment; same answer in both CTAs
        if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, kStatusTimeout | (15 << 8));
        return;
    }
    uint64_t* bars = reinterpret_cast<uint64_t*>(tiles + L::kTileBytes);
    uint64_t* kfull = bars;
    uint64_t* kempty = kfull + L::kNK;
    uint64_t* vfull = kempty + L::kNK;
    uint64_t* vempty = vfull + L::kNV;
    uint64_t* q_full = vempty + L::kNV;  // leader only: both CTAs' query rows are written
    uint64_t* o_free = q_full + 1;     // leader only: both CTAs' softmax warps have read O of a piece
    uint64_t* epi_done = o_free + 1;   // this CTA's output staging (P + V ring) is free again
    uint64_t* s_full = epi_done + 1;   // [2]
    uint64_t* p_ready = s_full + 2;    // [2] leader only: one arrival per softmax warp of the pair
    uint64_t* pv_done = p_ready + 2;   // [2]
    uint64_t* fin = pv_done + 2;       // the final partial-sum exchange of a piece
    uint64_t* sc_full = fin + 1;       // [kScaleTiles] the tile's page scales are there
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::kNumBars);
    volatile int32_t* abort_flag = reinterpret_cast<volatile int32_t*>(tmem_slot + 1);
    float4* page_scales = reinterpret_cast<float4*>(tiles + L::kOffScale);
    float* row_scale = reinterpret_cast<float*>(tiles + L::kOffRow);
    float* sm_max = reinterpret_cast<float*>(tiles + L::kOffMax);  // [4][64] partial maxima of a raise
    // [4][64] final partial sums; a raise ends in a barrier behind its reads of sm_max, so a warp that leaves the tile loop may write
    // them, and the next piece's first raise comes behind epi_done, i.e. behind every warp's reads of the sums
    float* sm_l = sm_max;

    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t cta = cluster_ctarank();  // 0 = leader
    const Abort ab{abort_flag, p.status};

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kNumBars; ++i) {
            uint64_t* bar = &bars[i];
            const bool pair_wide = bar == &p_ready[0] || bar == &p_ready[1] || bar == o_free || bar == q_full;
            const bool cta_wide = bar == fin || bar == epi_done;
            mbar_init(bar, pair_wide ? 2 * L::kSoftmaxWarps : (cta_wide ? L::kSoftmaxWarps : 1));
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc2(tmem_slot, 512);
        tmem_relinquish2();
    }

    pdl_launch_dependents();
    if (warp == 0 && elect_one()) {
        tma_prefetch_desc(&tmC);
        tma_prefetch_desc(&tmCr);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both CTAs' barriers exist before any remote arrival
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);
    pdl_wait();  // set-up is done (behind the preceding kernel's tail); everything below reads the caller's tensors
    // the plan of this pair: row block rb, and either one (sequence, split) piece or worker w's share
    const int pair = blockIdx.x >> 1;
    const int rb = pair % p.row_blocks;
    WholeOrBalanced walk;
    if (p.balanced) {
        walk.init_balanced(p.seqlens, p.B, p.S, pair / p.row_blocks, p.W, p.W, p.slack, reinterpret_cast<int32_t*>(sm_max), L::kThreads);
    } else {
        const int unit = pair / p.row_blocks;
        walk.init_fixed(p.seqlens, p.B, p.S, unit / p.S, unit % p.S);
    }
    const int rho0 = rb * 128 + (int)cta * 64;  // first (query, head) row of this CTA
    Piece pc;
    int pi = 0;  // non-empty pieces walked so far (phase of the per-piece barriers)

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer of the K ring, and the page
        // scales (both CTAs).  Every "full" barrier of the rings lives in the leader and counts the bytes of BOTH CTAs.
        const uint32_t e = elect_one();
        int ks = 0, n = 0;
        uint32_t kph = 1;  // parity that means "slot is free"
        bool ok = true;
        while (ok && warp_all(walk.next(pc))) {
            const int n_tiles = warp_uniform(pc.n_tiles);
            if (n_tiles == 0) continue;
            const int32_t T = p.seqlens[pc.b];
            // the query rows, which the softmax warps read when they are through with the piece before
            if (lane == 0 && rho0 < p.rows_total)
                prefetch_l2(reinterpret_cast<const uint8_t*>(p.q + ((int64_t)pc.b * p.rows_total + rho0) * 576),
                            (uint32_t)(p.rows_total - rho0 < 64 ? p.rows_total - rho0 : 64) * 1152u);
            // a lane looks up a run of 16 tokens of the tile: page numbers two tiles ahead, scales one
            PageWalk pw(p.rows, pc.b, (uint32_t)(pc.tok_begin + (lane & 7) * 16), T);
            auto scale_of = [&](int32_t page) { return (uint32_t)page < (uint32_t)p.n_pages ? p.page_scale[page] : 1.f; };
            int32_t page, page1, page2;
            uint32_t in_page, in_page1, in_page2;
            pw.next(page, in_page);
            pw.next(page1, in_page1);
            float cur = scale_of(page);
            for (int kt = 0; kt < n_tiles && ok; ++kt, ++n) {
                const int32_t row = page < 0 ? p.n_rows : (int32_t)((int64_t)page * p.rows.page_size + in_page);
                pw.next(page2, in_page2);
                const float next = scale_of(page1);
                int32_t y[NB];  // first cache rows of this CTA's half of the tile
#pragma unroll
                for (int rn = 0; rn < NB; ++rn) y[rn] = __shfl_sync(0xffffffffu, row, (int)cta * 4 + rn * (PG / 16));
#pragma unroll 1
                for (int kg = 0; kg < 2; ++kg) {
                    if (!(ok = warp_all(mbar_wait(&kempty[ks], kph, ab, 1)))) break;
                    if (kg == 0) {
                        if (lane < 8) {  // (the logarithm of a scale of zero would not be finite)
                            const float s = fmaxf(cur, 8.6736174e-19f);
                            page_scales[n % L::kScaleTiles * 8 + lane] = make_float4(cur, lg2(s), rcp(s), 0.f);
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sc_full[n % L::kScaleTiles]);
                    }
                    // group 0: latent boxes 0, 1;  group 1: latent boxes 2, 3 and the RoPE box
                    if (cta == 0) mbar_expect_tx(&kfull[ks], 2 * (2 * L::kBox + (kg == 1 ? L::kRBox : 0)), e);
                    __syncwarp();
                    const uint32_t bar = mapa(smem_u32(&kfull[ks]), 0);
                    uint8_t* dst = tiles + L::kOffK + ks * L::kKGroup;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int rn = 0; rn < NB; ++rn)
                            tma_load_2d_pair(dst + i * L::kBox + rn * PG * 128, &tmC, (2 * kg + i) * 128, y[rn], bar, e);
                    if (kg == 1) {
#pragma unroll
                        for (int rn = 0; rn < NB; ++rn) tma_load_2d_pair(dst + 2 * L::kBox + rn * PG * 64, &tmCr, 512, y[rn], bar, e);
                    }
                    if (++ks == L::kNK) { ks = 0; kph ^= 1; }
                }
                page = page1; in_page = in_page1;
                page1 = page2; in_page1 = in_page2;
                cur = next;
            }
            ++pi;
        }
    } else if (warp == L::kVProducerWarp) {
        // ------------------------------------------------------------------ TMA producer of the V ring (both
        // CTAs): the two rings fill independently of one another.  V groups in the order (tile, token half); a V slot is free
        // only after P.V of the previous tile, i.e. after Qh Kh^T of this tile has read the same cache rows
        // as K boxes, so the V boxes come out of L2.
        const uint32_t e = elect_one();
        int vs = 0;
        uint32_t vph = 1;
        bool ok = true;
        while (ok && warp_all(walk.next(pc))) {
            const int n_tiles = warp_uniform(pc.n_tiles);
            if (n_tiles == 0) continue;
            const int32_t T = p.seqlens[pc.b];
            PageWalk pw(p.rows, pc.b, (uint32_t)(pc.tok_begin + (lane & 7) * 16), T);
            // the V ring doubles as the output staging of the previous piece
            if (pi > 0 && !(ok = warp_all(mbar_wait(epi_done, (pi - 1) & 1, ab, 16)))) break;
            int32_t page, page1;
            uint32_t in_page, in_page1;
            pw.next(page, in_page);
            for (int vt = 0; vt < n_tiles && ok; ++vt) {
                const int32_t row = page < 0 ? p.n_rows : (int32_t)((int64_t)page * p.rows.page_size + in_page);
                pw.next(page1, in_page1);
#pragma unroll 1
                for (int vh = 0; vh < 2; ++vh) {
                    const int32_t left = T - (pc.tok_begin + vt * 128 + vh * 64);
                    const int cut = (int)warp_uniform((uint32_t)cut_run<PG>(left, 64));
                    if (!(ok = warp_all(mbar_wait(&vempty[vs], vph, ab, 2)))) break;
                    if (cta == 0) mbar_expect_tx(&vfull[vs], 2 * L::kVGroup, e);
                    __syncwarp();
                    const uint32_t bar = mapa(smem_u32(&vfull[vs]), 0);
                    uint8_t* dst = tiles + L::kOffV + vs * L::kVGroup;
                    int32_t y[NB];
#pragma unroll
                    for (int rn = 0; rn < NB; ++rn) y[rn] = __shfl_sync(0xffffffffu, row, vh * 4 + rn * (PG / 16));
                    // box m: latent columns [256m + 128cta, +128) -- this CTA's half of MMA m's N
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int rn = 0; rn < NB; ++rn)
                            tma_load_2d_pair(dst + m * L::kBox + rn * PG * 128, &tmC, 256 * m + 128 * (int)cta, y[rn], bar, rn != cut ? e : 0u);
                    if (cut >= 0)
                        load_cut_run<PG, 2>(cut_maps, lane, left % PG, __shfl_sync(0xffffffffu, row, vh * 4 + cut * (PG / 16)), p.n_rows,
                                            [&](const CUtensorMap* map, int m, int r, int32_t yy) {
                                                tma_load_2d_pair(dst + m * L::kBox + (cut * PG + r) * 128, map, 256 * m + 128 * (int)cta, yy, bar);
                                            });
                    if (++vs == L::kNV) { vs = 0; vph ^= 1; }
                }
                page = page1; in_page = in_page1;
            }
            ++pi;
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (leader CTA only)
        if (cta == 0) {
            const uint32_t e = elect_one();
            constexpr uint32_t idesc_qk = idesc_e4m3(128, 128, 0, 0);
            constexpr uint32_t idesc_pv[2] = {idesc_e4m3(128, 256, 0, 1), idesc_e4m3(128, 256, 0, 1) | (1u << 7)};  // P: E4M3, E5M2
            const uint32_t q_lo = desc_lo(desc_kmajor_sw128(smem_u32(tiles)));
            const uint32_t qr_lo = desc_lo(desc_kmajor_sw64(smem_u32(tiles + 4 * L::kBox)));
            const uint32_t p_lo = desc_lo(desc_kmajor_sw128(smem_u32(tiles + L::kOffP)));
            int ks = 0, vs = 0;
            uint32_t kph = 0, vph = 0;
            int gt = 0;  // tiles issued so far: score buffer = gt & 1, phase = (gt >> 1) & 1
            auto issue_qk = [&](int n) -> bool {
                const uint32_t d = tmem_base + kA8ColS + (uint32_t)(n & 1) * 64;
#pragma unroll 1
                for (int g2 = 0; g2 < 2; ++g2) {
                    if (!warp_all(mbar_wait_fast(&kfull[ks], kph, ab, 3))) return false;
                    tc_fence_after();
                    const uint32_t kd = desc_lo(desc_kmajor_sw128(smem_u32(tiles + L::kOffK + ks * L::kKGroup)));
                    const uint32_t qd = q_lo + ((g2 * 2 * L::kBox) >> 4);
                    if (g2 == 0)
                        umma_f8_ss2_lo<false>(d, qd, kd, idesc_qk, kDescHiSw128, e);  // the tile's first MMA overwrites S
                    else
                        umma_f8_ss2_lo<true>(d, qd, kd, idesc_qk, kDescHiSw128, e);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                if ((term | i | kk) != 0)
                                    umma_f8_ss2_lo<true>(d, qd + ((term * L::kQTerm + i * L::kBox + kk * 32) >> 4),
                                                         kd + ((i * L::kBox + kk * 32) >> 4), idesc_qk, kDescHiSw128, e);
                    if (g2 == 1) {  // the RoPE part: 64 elements = 2 x 32, 64-byte swizzle
                        const uint32_t krd = desc_lo(desc_kmajor_sw64(smem_u32(tiles + L::kOffK + ks * L::kKGroup + 2 * L::kBox)));
#pragma unroll
                        for (int term = 0; term < 2; ++term)
#pragma unroll
                            for (int kk = 0; kk < 2; ++kk)
                                umma_f8_ss2_lo<true>(d, qr_lo + ((term * L::kQTerm + kk * 32) >> 4), krd + ((kk * 32) >> 4), idesc_qk,
                                                     kDescHiSw64, e);
                    }
                    umma_commit2(&kempty[ks], 3, e);
                    if (++ks == L::kNK) { ks = 0; kph ^= 1; }
                }
                umma_commit2(&s_full[n & 1], 3, e);
                return true;
            };
            bool ok = true;
            while (ok && warp_all(walk.next(pc))) {
                const int n_tiles = warp_uniform(pc.n_tiles);
                if (n_tiles == 0) continue;
                if (!(ok = warp_all(mbar_wait(q_full, pi & 1, ab, 4)))) break;
                tc_fence_after();
                if (!(ok = issue_qk(gt))) break;
                for (int t = 0; t < n_tiles && ok; ++t) {
                    const int n = gt + t;
                    if (t + 1 < n_tiles && !(ok = issue_qk(n + 1))) break;
                    if (!(ok = warp_all(mbar_wait_fast(&p_ready[n & 1], (n >> 1) & 1, ab, 5)))) break;
                    // the first P.V of a piece overwrites O: the previous piece's O must have been read
                    if (t == 0 && pi > 0 && !(ok = warp_all(mbar_wait(o_free, (pi - 1) & 1, ab, 14)))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = warp_all(mbar_wait_fast(&vfull[vs], vph, ab, 6)))) break;
                        tc_fence_after();
                        // V box m: [64 tokens x 128 latent columns], MN-major; a k-step is 32 token rows (4 KB)
                        const uint32_t vd = desc_lo(desc_mnmajor_sw128(smem_u32(tiles + L::kOffV + vs * L::kVGroup), L::kBox));
                        const uint32_t pd = p_lo + ((h * 64) >> 4);  // tokens [64h, 64h + 64) of the P rows
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const uint32_t dm = tmem_base + kA8ColO + (uint32_t)m * 128;
#pragma unroll
                            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                                for (int term = 0; term < 2; ++term) {
                                    const uint32_t pa = pd + ((term * L::kPTerm + kk * 32) >> 4), va = vd + ((m * L::kBox + kk * 4096) >> 4);
                                    if ((kk | term) == 0 && (t | h) == 0)
                                        umma_f8_ss2_lo<false>(dm, pa, va, idesc_pv[term], kDescHiSw128, e);  // first P.V of a piece
                                    else
                                        umma_f8_ss2_lo<true>(dm, pa, va, idesc_pv[term], kDescHiSw128, e);
                                }
                        }
                        umma_commit2(&vempty[vs], 3, e);
                        if (++vs == L::kNV) { vs = 0; vph ^= 1; }
                    }
                    if (ok) umma_commit2(&pv_done[n & 1], 3, e);
                }
                gt += n_tiles;
                ++pi;
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax
        const int q = warp & 3;              // TMEM lane quadrant this warp may access
        const int ch = (warp - 2) >> 2;      // which 32 of the lane's 64 score columns
        const int Lr = q * 32 + lane;        // TMEM lane
        const int r = Lr & 63;               // row within this CTA
        const int hf = Lr >> 6;              // token half of each 128-token tile / column half of each O block
        const int part = hf * 2 + ch;        // one of the four threads of row r
        const int rho = rho0 + r;            // (query, head) row of the sequence
        const bool row_valid = rho < p.rows_total;
        const int pq = row_valid ? rho / p.h_q : 0;
        const uint32_t lane_base = tmem_base + ((uint32_t)(q * 32) << 16);
        const uint32_t p_ready_l[2] = {mapa(smem_u32(&p_ready[0]), 0), mapa(smem_u32(&p_ready[1]), 0)};
        const uint32_t o_free_l = mapa(smem_u32(o_free), 0), q_full_l = mapa(smem_u32(q_full), 0);
        const float scale_abs = fabsf(p.scale_log2);  // (a negative softmax scale turns the queries' signs)
        int gt = 0;  // tiles walked so far

        // The query rows of a piece, eight a warp, a pair at a time with the next pair on its way.
        auto write_q = [&]() {
            // (the warp's number anew: what follows from it is not to be worked out ahead and kept in registers over the tiles)
            int sw = warp - 2;
            asm volatile("" : "+r"(sw));
            auto fetch = [&](QueryPair<576>& rows, int i) {
                const int rr = rho0 + sw * 8 + 2 * i + (lane >> 4);
                rows.fetch(p.q + ((int64_t)pc.b * p.rows_total + rr) * 576, rr < p.rows_total, lane);
            };
            QueryPair<576> rows, ahead;
            fetch(rows, 0);
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                if (i < 3) fetch(ahead, i + 1);
                const int rl = sw * 8 + 2 * i + (lane >> 4);
                const float qs = rows.cut(lane, p.scale_log2, [&](int col, const uint2& hi, const uint2& lo) {
                    // boxes of 128 columns: 128-byte rows, 16-byte chunks XORed with r % 8; the RoPE box: 64-byte rows, with r / 2 % 4
                    const int blk = col / 128;
                    uint8_t* at = tiles + blk * L::kBox + (col & 8) +
                                  (blk < 4 ? rl * 128 + ((((col % 128) >> 4) ^ (rl & 7)) << 4) : rl * 64 + ((((col - 512) >> 4) ^ ((rl >> 1) & 3)) << 4));
                    *reinterpret_cast<uint2*>(at) = hi;
                    *reinterpret_cast<uint2*>(at + L::kQTerm) = lo;
                });
                if (lane % 16 == 0) row_scale[rl] = scale_abs * qs;
                rows = ahead;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(q_full_l);
        };

        while (walk.next(pc)) {
            GQLA_DEBUG_CHECK(pc.b >= 0 && pc.b < p.B, p.status, 32);  // a piece names a sequence of the batch
            const int32_t T = p.seqlens[pc.b];
            const int64_t slot0 = (int64_t)pc.b * p.S;
            GQLA_DEBUG_CHECK(pc.n_tiles == 0 || (pc.k >= 0 && pc.k < p.S), p.status, 33);  // ... and one of its S slots
            GQLA_DEBUG_CHECK(pc.tok_begin >= 0 && pc.tok_begin <= pc.tok_end && pc.tok_end <= (T > 0 ? T : 0), p.status, 34);
            GQLA_DEBUG_CHECK(pc.n_tiles == (pc.tok_end > pc.tok_begin ? (pc.tok_end - pc.tok_begin + 127) / 128 : 0), p.status, 35);
            GQLA_DEBUG_CHECK(!p.balanced || pc.tok_begin % 128 == 0, p.status, 36);  // balanced pieces start on tile boundaries
            GQLA_DEBUG_CHECK(pc.fill_begin >= 0 && pc.fill_begin <= pc.fill_end && pc.fill_end <= p.S || pc.fill_end == 0, p.status, 37);
            // split slots this worker marks empty
            if (part == 0 && row_valid)
                for (int kk = pc.fill_begin; kk < pc.fill_end; ++kk) p.lse_part[(slot0 + kk) * p.rows_total + rho] = -INFINITY;
            if (pc.n_tiles == 0 && p.balanced) continue;  // an empty sequence: its slots were marked above
            int32_t lim = visible_limit(T, p.s_q, pq);
            if (lim > pc.tok_end) lim = pc.tok_end;
            lim -= pc.tok_begin;
            if (!row_valid) lim = 0;
            // (the scores of the previous piece's last tile have been read, so nothing reads its rows any more)
            if (pc.n_tiles > 0) write_q();
            named_bar_sync(1, L::kSoftmaxWarps * 32);  // the scales are there
            const float sl2 = row_scale[r];
            // m_used: the row's softmax REFERENCE (log2 units), the same in the four threads of the row: a raise puts it kAF8Bias
            // binades below the row's maximum so far, and the next raise comes when a score exceeds it by more than kAF8Grow
            // (P' <= 430, E4M3 reaches 448).
            float m_used = -INFINITY, l = 0.f;
            bool ok = true;

            for (int t = 0; t < pc.n_tiles && ok; ++t) {
                const int n = gt + t;
                const int sb = n & 1;
                const uint32_t nph = (n >> 1) & 1;
                // a failed wait raises the CTA's abort flag; the warps agree on leaving at the barrier below
                bool okl = __all_sync(0xffffffffu, mbar_wait_fast(&s_full[sb], nph, ab, 7));
                tc_fence_after();
                const int tok0 = t * 128 + hf * 64 + ch * 32;
                if (okl) okl = __all_sync(0xffffffffu, mbar_wait_fast(&sc_full[n % L::kScaleTiles], n / L::kScaleTiles & 1, ab, 10));
                const float4 ps[2] = {page_scales[n % L::kScaleTiles * 8 + part * 2], page_scales[n % L::kScaleTiles * 8 + part * 2 + 1]};
                const float sa[2] = {sl2 * ps[0].x, sl2 * ps[1].x};
                uint32_t x[32];
                if (okl) {
                    tmem_ld32(lane_base + kA8ColS + (uint32_t)sb * 64 + ch * 32, x);
                    tmem_wait_ld();
                }
                const bool full = tok0 + 32 <= lim;  // every score of this thread is visible
                float mx[2] = {-INFINITY, -INFINITY};  // of the first and the last 16 tokens
                if (okl) {
                    if (full) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) mx[c / 16] = fmaxf(mx[c / 16], __uint_as_float(x[c]));
                    } else {
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (tok0 + c < lim) mx[c / 16] = fmaxf(mx[c / 16], __uint_as_float(x[c]));
                    }
                }
                // Does any score of the CTA outgrow its row's reference?  One barrier.red instead of an exchange of the
                // row maxima (the other three parts of a row live in other warps); only then are the maxima exchanged.
                const float m_t = fmaxf(fmaf(mx[0], sa[0], ps[0].y), fmaf(mx[1], sa[1], ps[1].y));
                float factor = 1.f;
                bool need = false;
                if (vote_any(1, m_t > m_used + kAF8Grow || !okl, L::kSoftmaxWarps * 32)) {
                    float* mxs = sm_max;
                    mxs[part * 64 + r] = m_t;
                    if (vote_any(1, !okl, L::kSoftmaxWarps * 32)) { ok = false; break; }  // leaving is agreed on (tc_common.cuh)
                    const float row_max = fmaxf(fmaxf(mxs[r], mxs[64 + r]), fmaxf(mxs[128 + r], mxs[192 + r]));
                    const float m_new = fmaxf(m_used, row_max - kAF8Bias);
                    need = m_new > m_used;
                    factor = need ? ex2(m_used - m_new) : 1.f;  // ex2(-inf) = 0 on first use
                    if (need) {
                        l *= factor;
                        m_used = m_new;
                    }
                    named_bar_sync(1, L::kSoftmaxWarps * 32);  // the maxima may be rewritten by the next raise
                }
                const float m_sub = m_used == -INFINITY ? 0.f : m_used;
                uint32_t pk[2][8];  // [term]
                const float up[2] = {ps[0].y - m_sub, ps[1].y - m_sub};
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const int h2 = c / 16;
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e[i] = ex2(fmaf(__uint_as_float(x[c + i]), sa[h2], up[h2]));
                        if (!full && !(okl && tok0 + c + i < lim)) e[i] = 0.f;
                        sum[h2] += e[i];
                    }
                    uint16_t h0, h1, l0, l1;
                    split_e4m3_e5m2(e[0], e[1], h0, l0);
                    split_e4m3_e5m2(e[2], e[3], h1, l1);
                    pk[0][c / 4] = (uint32_t)h0 | ((uint32_t)h1 << 16);
                    pk[1][c / 4] = (uint32_t)l0 | ((uint32_t)l1 << 16);
                }
                l = fmaf(sum[0], ps[0].z, fmaf(sum[1], ps[1].z, l));
                // O may be rescaled, and the P buffer rewritten, only once P.V(n-1) has completed
                if (t > 0 && okl) {
                    okl = __all_sync(0xffffffffu, mbar_wait_fast(&pv_done[(n - 1) & 1], ((n - 1) >> 1) & 1, ab, 8));
                    tc_fence_after();
                }
                if (__any_sync(0xffffffffu, need) && t > 0 && okl) {
                    // this thread's share of the lane's O: columns [128m + 64ch, +64) for m = 0, 1
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t col = kA8ColO + (uint32_t)(c >> 1) * 128 + ch * 64 + (c & 1) * 32;
                        uint32_t o[32];
                        tmem_ld32(lane_base + col, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
                        tmem_st32(lane_base + col, o);
                    }
                    tmem_wait_st();
                }
                // P row r: 128 bytes = 128 tokens = 8 chunks of 16 E4M3, chunk index XORed with (r & 7); this
                // thread's 32 tokens are chunks 4 hf + 2 ch and the next one
                uint8_t* prow = tiles + L::kOffP + r * 128;
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                    for (int c2 = 0; c2 < 2; ++c2)
                        *reinterpret_cast<uint4*>(prow + term * L::kPTerm + (((hf * 4 + ch * 2 + c2) ^ (r & 7)) << 4)) =
                            make_uint4(pk[term][4 * c2], pk[term][4 * c2 + 1], pk[term][4 * c2 + 2], pk[term][4 * c2 + 3]);
                fence_proxy_async_smem();  // generic-proxy writes of P -> visible to the tensor core
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && okl) mbar_arrive_cluster(p_ready_l[sb]);  // withheld after a failed wait: the next vote ends the loop
            }

            // -------------------------------------------------------------- epilogue: normalise and store
            const int n_tiles = pc.n_tiles, out_k = pc.k;
            const int64_t out_row = (slot0 + pc.k) * p.rows_total + rho;
            sm_l[part * 64 + r] = l;
            const int n_last = gt + n_tiles - 1;
            if (n_tiles > 0 && ok)
                ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[n_last & 1], (n_last >> 1) & 1, ab, 9));
            tc_fence_after();
            __syncwarp();
            if (lane == 0) mbar_arrive(fin);
            if (!__all_sync(0xffffffffu, mbar_wait(fin, pi & 1, ab, 11))) ok = false;
            const float Lt = (sm_l[r] + sm_l[64 + r]) + (sm_l[128 + r] + sm_l[192 + r]);
            const bool live = ok && n_tiles > 0 && Lt != 0.f;  // the row sees something (a NaN sum is something)
            const float inv = live ? 1.f / Lt : 0.f;
            // The output rows leave through shared memory (P and the V ring are idle now: the last P.V has completed): every warp turns 32
            // rows x 64 columns of MMA m's block by itself and stores two rows of 256 bytes at a time.  (As bulk stores of 256 bytes, of
            // which a CTA has 512, a piece's output took 8000 cycles.)  The padded pitch keeps the 16-byte accesses of a quarter warp on
            // distinct banks.
            {
                uint8_t* own = tiles + L::kOffP + (warp - 2) * 32 * L::kWarpPitch;
                const int64_t row0 = (slot0 + out_k) * p.rows_total + rho0 + (q & 1) * 32;  // the warp's first row
                const int rows_left = p.rows_total - rho0 - (q & 1) * 32;
#pragma unroll 1
                for (int m = 0; m < 2; ++m) {
#pragma unroll 1
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t o[32];
                        if (n_tiles > 0 && ok) {  // warp-uniform
                            tmem_ld32(lane_base + kA8ColO + m * 128 + ch * 64 + c, o);
                            tmem_wait_ld();
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            reinterpret_cast<float4*>(own + lane * L::kWarpPitch)[c / 4 + i] =
                                live ? make_float4(__uint_as_float(o[4 * i]) * inv, __uint_as_float(o[4 * i + 1]) * inv,
                                                   __uint_as_float(o[4 * i + 2]) * inv, __uint_as_float(o[4 * i + 3]) * inv)
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    if (m == 1) {  // O has been read: the next piece's first P.V may overwrite it
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(o_free_l);
                    }
                    __syncwarp();
                    float* out = p.o_part + row0 * 512 + 256 * m + 128 * hf + 64 * ch + (lane & 15) * 4;
#pragma unroll 4
                    for (int i = lane >> 4; i < 32; i += 2)
                        if (i < rows_left && ok)
                            *reinterpret_cast<float4*>(out + (int64_t)i * 512) = reinterpret_cast<const float4*>(own + i * L::kWarpPitch)[lane & 15];
                    __syncwarp();
                }
            }
            // staging (and with it P and the V ring) is free again once every warp's stores have read it
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(epi_done);
            if (!__all_sync(0xffffffffu, mbar_wait(epi_done, pi & 1, ab, 12))) ok = false;
            if (row_valid && part == 0)
                p.lse_part[out_row] =
                    live ? (m_used + log2f(Lt)) * 0.6931471805599453f : -INFINITY;
            gt += n_tiles;
            ++pi;
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // neither CTA leaves while the other may still signal its barriers
    if (warp == 1) tmem_dealloc2(tmem_base, 512);
}

}  // namespace tc
}  // namespace gqla
