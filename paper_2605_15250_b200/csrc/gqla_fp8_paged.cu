// C-ABI entry points of the cache append with position rotation and of attention over E4M3 pages with a scale per page
// and head: argument validation, kernel selection, launch.
#include "../../include/gqla.h"

#include <algorithm>
#include <type_traits>

#include "append_rope.cuh"
#include "common.cuh"
#include "sched.cuh"
#include "tc_common.cuh"
#include "tc_decode_fp8_pair.cuh"
#include "tc_decode_fp8_paged.cuh"

using namespace gqla;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

gqla_status check_dims(const gqla_dims* d) {
    if (d == nullptr) return GQLA_ERR_NULL;
    if (d->h_q <= 0 || d->g <= 0 || d->d_h <= 0 || d->r_kv <= 0 || d->d_r < 0 || d->h_q % d->g != 0) return GQLA_ERR_SHAPE;
    return GQLA_OK;
}

// ------------------------------------------------------------------------------------------------ appending

struct AppendCall {
    gqla_dtype dtype;
    int32_t B;
    int64_t n;
    const int32_t *new_start, *seqlens;
    const void* k_r;
    int64_t k_r_stride;
    const float* rope;
    int32_t rope_rows;
    gqla_rope_style style;
    const void* q_r;
    int64_t q_tok, q_head;
    void* q_out;
    int64_t o_tok, o_head;
};

// What the three append calls check alike (null pointers too; n == 0 is nothing to do and checked by the caller first).
gqla_status check_append(const gqla_dims* d, const AppendCall& a) {
    gqla_status s = check_dims(d);
    if (s != GQLA_OK) return s;
    if (a.dtype != GQLA_BF16 && a.dtype != GQLA_F32) return GQLA_ERR_DTYPE;
    if (d->d_r % 2 != 0 || a.B < 0 || a.n < 0 || a.n > 0x7fffffffLL || (a.style != GQLA_ROPE_PAIRS && a.style != GQLA_ROPE_HALVES))
        return GQLA_ERR_SHAPE;
    if (a.B == 0 || a.n == 0) return GQLA_OK;
    if (a.new_start == nullptr || a.seqlens == nullptr || (a.q_r == nullptr) != (a.q_out == nullptr)) return GQLA_ERR_NULL;
    if (d->d_r > 0 && (a.k_r == nullptr || a.rope == nullptr)) return GQLA_ERR_NULL;
    if (d->d_r > 0 && (a.k_r_stride < d->d_r || a.rope_rows < 0)) return GQLA_ERR_SHAPE;
    if (a.q_r != nullptr && (a.q_head < d->d_r || a.o_head < d->d_r || a.q_tok < d->d_r || a.o_tok < d->d_r)) return GQLA_ERR_SHAPE;
    return GQLA_OK;
}

// Whether sixteen-byte accesses of eight elements cover the rows: strides, widths and pointers.
bool vectors(const gqla_dims& d, const AppendCall& a) {
    return d.d_r % 16 == 0 && a.k_r_stride % 8 == 0 && aligned(a.k_r, 16) && aligned(a.rope, 16) &&
           (a.q_r == nullptr || (aligned(a.q_r, 16) && aligned(a.q_out, 16) && a.q_tok % 8 == 0 && a.q_head % 8 == 0 &&
                                 a.o_tok % 8 == 0 && a.o_head % 8 == 0));
}

template <typename Args>
void fill(Args& k, const gqla_dims& d, const AppendCall& a) {
    k.nr = NewRows{a.B, a.n, a.new_start, a.seqlens};
    k.rope = RopeTable{a.rope, a.rope_rows, d.d_r, a.style == GQLA_ROPE_HALVES};
    k.q = QueryRows{a.q_r, a.q_out, a.q_tok, a.q_head, a.o_tok, a.o_head, d.h_q};
    k.k_r = a.k_r;
    k.k_r_stride = a.k_r_stride;
}

int64_t query_blocks(const gqla_dims& d, const AppendCall& a, bool vec, int threads) {
    if (a.q_r == nullptr || d.d_r == 0) return 0;
    const int64_t items = a.n * d.h_q * (vec ? RopeItem<8>::count(d.d_r) : RopeItem<1>::count(d.d_r));
    return (items + threads - 1) / threads;
}

template <typename Args>
gqla_status launch_append(void (*kern)(Args), const Args& a, int64_t blocks, int threads, cudaStream_t st, int smem = 0) {
    if (blocks > 0x7fffffffLL) return GQLA_ERR_SHAPE;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
        return GQLA_ERR_CUDA;
    return tc::launch_pdl(kern, dim3((unsigned)blocks), dim3(threads), smem, st, a) == cudaSuccess ? GQLA_OK : GQLA_ERR_CUDA;
}

template <int THREADS>
gqla_status launch_append_fp8_of(gqla_dtype dtype, bool vec, const AppendFp8Args& a, int64_t blocks, cudaStream_t st) {
    if (dtype == GQLA_BF16)
        return vec ? launch_append(append_fp8_kernel<__nv_bfloat16, true, THREADS>, a, blocks, THREADS, st,
                                   a.held * HeldChunks<__nv_bfloat16, true, THREADS>::kBytes)
                   : launch_append(append_fp8_kernel<__nv_bfloat16, false, THREADS>, a, blocks, THREADS, st);
    return launch_append(vec ? append_fp8_kernel<float, true, THREADS> : append_fp8_kernel<float, false, THREADS>, a, blocks, THREADS, st);
}

gqla_status launch_append_fp8(const gqla_dims& d, const AppendCall& call, AppendFp8Args& a, bool vec, const int32_t* block_table,
                              int32_t max_pages, int32_t page_size, int64_t n_rows, int32_t* status_word, cudaStream_t st) {
    fill(a, d, call);
    a.block_table = block_table; a.max_pages = max_pages; a.page_size = page_size; a.status = status_word;
    a.n_pages = (int32_t)(n_rows / page_size);
    for (Fp8Plane& p : a.plane) {
        const int turned = p.rope_heads ? (vec ? RopeItem<4>::count(d.d_r) : RopeItem<1>::count(d.d_r)) : 0;
        const int width = p.a_width + (p.rope_heads ? d.d_r : 0), each = vec ? 8 : 1;
        p.copied = ItemsOfRow(std::max(p.a_width / each, 1));
        p.turned = ItemsOfRow(std::max(turned, 1));
        p.coded = ItemsOfRow(std::max(width / each, 1));
    }
    a.heads_in_all = a.plane[0].heads + a.plane[1].heads + a.plane[2].heads;
    int shift = 0;
    while (((int64_t)2 << shift) <= page_size) ++shift;  // 2^shift <= page_size < 2^(shift + 1)
    const int64_t by_pages = (call.n >> shift) + 2 * (int64_t)call.B;
    const int64_t units = call.n < by_pages ? call.n : by_pages;
    a.unit_shift = call.n < by_pages ? -1 : shift;
    // a unit by rows has a row or a few: room for one chunk a thread leaves that of the next launch's blocks free, which then start
    // early (64 rows into 17 planes' heads, launches back to back, 128 threads: 7.2 us with room for eight chunks, 5.8 with room for one)
    a.held = call.n < by_pages ? 1 : 16;
    if (units > 0x7fffffffLL) return GQLA_ERR_SHAPE;
    a.kv_blocks = units * a.heads_in_all;
    const int threads = a.heads_in_all == 1 ? kLatentThreads : kPlaneThreads;
    const int64_t blocks = a.kv_blocks + query_blocks(d, call, vec, threads);
    return threads == kLatentThreads ? launch_append_fp8_of<kLatentThreads>(call.dtype, vec, a, blocks, st)
                                     : launch_append_fp8_of<kPlaneThreads>(call.dtype, vec, a, blocks, st);
}

// ------------------------------------------------------------------------------------------------ attention

struct Fp8PagedCall {
    const gqla_dims* d;
    gqla_dtype dtype;
    int32_t B, s_q;
    float scale;
    int32_t S;
    const void* q;
    const uint8_t *k, *v, *k_r;         // absorb path: k alone
    int64_t k_stride, k_r_stride;       // bytes between rows of k (absorb path) and of k_r
    int64_t n_rows;
    const float *k_scale, *v_scale, *r_scale;
    const int32_t* block_table;
    int32_t max_pages, page_size;
    const int32_t* seqlens;
    float *o_part, *lse_part;
    int32_t* status;
    bool latent;
};

// Any dimensions, any page size, bf16 or fp32 queries: one warp per (sequence, split, position, head) row, fp32 throughout.  Bound by its
// instructions, a load and a decoding per code and head: 8 x 1024 rows, 32 heads, eight splits, fp32 queries 290 us on the absorb path, 221 on
// the GQA path.
struct Fp8PagedGeneric {
    const void* q;
    const e4m3 *kA, *kB, *v;
    int64_t kA_stride, kB_stride, v_stride;
    int32_t dA, dB, dv, kv_heads;  // kv_heads: g on the GQA path, 1 on the absorb path
    const float *sA, *sB, *sV;
    RowMap rows;
    int32_t n_pages;
    const int32_t* seqlens;
    int32_t B, S, s_q, h_q;
    float scale;
    float *o_part, *lse_part;
    int32_t* status;
};

constexpr int kGenericCols = 16;  // value columns per lane: dv <= 512

template <typename TQ>
__global__ void __launch_bounds__(128) decode_fp8_paged_generic_kernel(const Fp8PagedGeneric a) {
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= (int64_t)a.B * a.S * a.s_q * a.h_q) return;
    const int i = (int)(row % a.h_q), p = (int)(row / a.h_q % a.s_q);
    const int k = (int)(row / ((int64_t)a.h_q * a.s_q) % a.S), b = (int)(row / ((int64_t)a.h_q * a.s_q * a.S));
    const int j = i / (a.h_q / a.kv_heads);
    const int32_t T = a.seqlens[b];
    int32_t begin, end;
    split_range(T, a.S, k, &begin, &end);
    const int32_t lim = visible_limit(T, a.s_q, p);
    if (end > lim) end = lim;
    const TQ* q = (const TQ*)a.q + ((int64_t)(b * a.s_q + p) * a.h_q + i) * (a.dA + a.dB);
    float scale = 0.f;  // NaN if an element of the query is no number or infinite: so are all scores of the row then, as on the tensor core
    for (int d = lane; d < a.dA + a.dB; d += 32) scale = fmaf(ldf(q + d), 0.f, scale);
    scale = warp_sum(scale) + a.scale;
    float acc[kGenericCols];
#pragma unroll
    for (int c = 0; c < kGenericCols; ++c) acc[c] = 0.f;
    float m = -FLT_MAX, l = 0.f;  // (a score of -inf weighs nothing; a NaN, which fmaxf passes over, makes the sum NaN)
    int32_t page = -1;
    float sA = 1.f, sB = 0.f, sV = 1.f;
    for (int32_t s = begin; s < end; ++s) {
        if (s == begin || s % a.rows.page_size == 0) {
            const int32_t kk = s / a.rows.page_size;
            page = kk < a.rows.max_pages ? a.rows.block_table[(int64_t)b * a.rows.max_pages + kk] : -1;
            if ((uint32_t)page >= (uint32_t)a.n_pages) {  // a page outside the cache: its tokens are left out
                if (lane == 0) append_error(a.status, 2);
                page = -1;
            } else {
                sA = a.sA[(int64_t)page * a.kv_heads + j];
                sV = a.sV[(int64_t)page * a.kv_heads + j];
                if (a.dB > 0) sB = a.sB[page];
            }
        }
        if (page < 0) continue;
        const int64_t n = (int64_t)page * a.rows.page_size + s % a.rows.page_size;
        const e4m3* ka = a.kA + n * a.kA_stride + (int64_t)j * a.dA;
        float dA = 0.f, dB = 0.f;
        for (int d = lane; d < a.dA; d += 32) dA = fmaf(ldf(q + d), ldf(ka + d), dA);
        for (int d = lane; d < a.dB; d += 32) dB = fmaf(ldf(q + a.dA + d), ldf(a.kB + n * a.kB_stride + d), dB);
        const float x = warp_sum(fmaf(dA, sA, dB * sB)) * scale;
        const float m_new = fmaxf(m, x);
        const float corr = expf(m - m_new);
        const float e = expf(x - m_new);
        l = l * corr + e;
        const float w = e * sV;
        const e4m3* vr = a.v + n * a.v_stride + (int64_t)j * a.dv;
#pragma unroll
        for (int c = 0; c < kGenericCols; ++c) {
            const int d = lane + 32 * c;
            if (d < a.dv) acc[c] = fmaf(w, ldf(vr + d), acc[c] * corr);
        }
        m = m_new;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // (nothing visible)
#pragma unroll
    for (int c = 0; c < kGenericCols; ++c) {
        const int d = lane + 32 * c;
        if (d < a.dv) a.o_part[row * a.dv + d] = acc[c] * inv;
    }
    if (lane == 0) a.lse_part[row] = l == 0.f ? -INFINITY : m + logf(l);
}

int pow2_at_least(int x) {
    int p = 1;
    while (p < x) p <<= 1;
    return p;
}

// How the query rows of a key head are cut into blocks of R = 16 or 32: hb heads (a power of two) by R / hb positions.
struct RowBlocks {
    int R, hb, n_hb, n_sb;
    int64_t count() const { return (int64_t)n_hb * n_sb; }
};
RowBlocks row_blocks(int32_t s_q, int32_t heads) {
    RowBlocks r;
    const int hp = pow2_at_least(heads < 32 ? heads : 32), sp = pow2_at_least(s_q < 32 ? s_q : 32);
    r.R = hp * sp <= 16 ? 16 : 32;
    r.hb = hp;
    if (hp * sp < r.R) r.hb = r.R / sp;  // padding heads fill the block
    r.n_hb = (heads + r.hb - 1) / r.hb;
    r.n_sb = (s_q + r.R / r.hb - 1) / (r.R / r.hb);
    return r;
}

bool covers(const gqla_dims& d, gqla_dtype dtype, int32_t s_q, int32_t page_size, bool latent) {
    return gqla_get_policy() == GQLA_POLICY_AUTO && dtype == GQLA_BF16 && d.d_r == 64 && (latent ? d.r_kv == 512 : d.d_h == 128) &&
           page_size % 16 == 0 && s_q <= 4096;
}

// Absorb path: CTA pairs with the query rows on M beyond 64 rows.  64 sequences of 4096 rows in a graph, on the tokens-on-M kernel and on
// pairs: 64 heads 66 and 80 us (half of a pair's rows are empty then), 72 heads 89 and 72, 40 heads at s_q = 2 110 and 73, 28 at 3 91 and
// 73, 32 at 3 93 and 74, 128 heads 115 and 77; 128 ragged ones of 256 to 4096 rows, 72 heads 125 and 112.
bool on_pairs(const gqla_dims& d, int32_t s_q, bool latent) { return latent && (int64_t)s_q * d.h_q > 64; }

// CTA pairs resident at once on the current device, 0 where it cannot be asked.
int resident_pairs() {
    static int cached[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (cached[dev] == 0) {
        auto kern = tc::decode_fp8_pair_kernel<64>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2 * 148, 1, 1);
        cfg.blockDim = dim3(tc::Fp8PairSmem::kThreads, 1, 1);
        cfg.dynamicSmemBytes = tc::Fp8PairSmem::kTotal;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, tc::Fp8PairSmem::kTotal) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            return 0;
        }
        cached[dev] = n;
    }
    return cached[dev];
}

int32_t token_workers(const gqla_dims& d, int32_t s_q, bool latent) {
    const RowBlocks r = row_blocks(s_q, latent ? d.h_q : d.h_q / d.g);
    const int64_t per = r.count() * (latent ? 1 : d.g);
    return per > 0 ? (int32_t)(sm_count() / per) : 0;
}
int32_t workers_of(const gqla_dims& d, int32_t s_q, bool latent) {
    if (on_pairs(d, s_q, latent)) return resident_pairs() / (int32_t)(((int64_t)s_q * d.h_q + 127) / 128);
    return token_workers(d, s_q, latent);
}

// Calls of few pieces stay off the pairs: with no more pieces than the tokens-on-M kernel has workers, each has a CTA of its own per 32
// rows, and twice the SMs of a pair work at its 128 rows.  Absorb path, 128 heads, on pairs and here: one sequence of 777 rows 16.9 and
// 15.7 us, of 4096 18.4 and 15.7; 4 of 1000 18.2 and 16.2; 32 of 128 18.2 and 15.2; in one piece each 32 of 2048 42.6 and 37.9, 32 of 8192
// 118 and 109.  (The cut is the same for any number of workers that is no less than the pieces: the share is then the longest sequence's,
// cut into S - 1.  Whether to cut at all goes by workers_of, which the caller knows: WholeOrBalanced.)
bool few_pieces(const Fp8PagedCall& c) {
    const int64_t pieces = (int64_t)c.B * (c.S < 0 ? -(int64_t)c.S - 1 : c.S);
    return pieces <= std::min(token_workers(*c.d, c.s_q, c.latent), c.S < 0 ? workers_of(*c.d, c.s_q, c.latent) : 0x7fffffff);
}

// Tiles by which the longest sequence may exceed a share for every sequence to be one piece.  Equal sequences of m tiles, cut and whole, us
// in a graph: absorb path, 100 of 32 heads (an excess of 0.32 m) m = 4 28.4 and 23.2, 9 36.3 and 31.5, 20 50.4 and 48.3; 50 of 128
// heads on pairs (also 0.32 m) 4 37.0 and 27.8, 18 56.0 and 50.3, 24 63.0 and 60.2, 32 71.7 and 72.6; GQA path, 14 of 32 heads (0.22 m)
// 8 19.0 and 15.4, 24 28.4 and 26.9, 32 32.8 and 32.1, 48 42.0 and 42.5.  With the excess at its bound, that is, whole sequences still win.
int32_t whole_slack(const gqla_dims& d, int32_t s_q, bool latent) { return latent && !on_pairs(d, s_q, latent) ? 3 : 6; }

template <int R, bool LATENT, int PG>
cudaError_t launch_tc(const tc::Fp8PagedParams& p, const CUtensorMap& k, const CUtensorMap& r, const CUtensorMap& v,
                      const tc::CutMaps<PG>& cut, unsigned grid, cudaStream_t st) {
    using L = tc::Fp8PagedSmem<R, LATENT>;
    auto kern = tc::decode_fp8_paged_kernel<R, LATENT, PG>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
    if (e != cudaSuccess) return e;
    return tc::launch_pdl(kern, dim3(grid), dim3(L::kThreads), L::kTotal, st, p, k, r, v, cut);
}

template <int PG>
gqla_status tc_decode_fp8_pairs(const Fp8PagedCall& c, cudaStream_t st) {
    const gqla_dims& d = *c.d;
    const int64_t rows_total = (int64_t)c.s_q * d.h_q, row_blocks = (rows_total + 127) / 128;
    const int32_t workers = c.S < 0 ? workers_of(d, c.s_q, true) : 0;
    const bool balanced = workers > 0;
    const int32_t S = c.S < 0 ? -c.S : c.S;
    const int64_t pairs = (balanced ? (int64_t)workers : (int64_t)c.B * S) * row_blocks;
    if (2 * pairs > 0x7fffffffLL || rows_total * c.B > 0x7fffffffLL) return GQLA_ERR_UNSUPPORTED;
    CUtensorMap tmC, tmCr;
    tc::CutMaps<PG> cut;
    const uint64_t dims[2] = {(uint64_t)(d.r_kv + d.d_r), (uint64_t)c.n_rows}, str[1] = {(uint64_t)c.k_stride};
    auto map = [&](CUtensorMap* m, uint32_t cols, uint32_t rows, CUtensorMapSwizzle swizzle) {
        const uint32_t box[2] = {cols, rows};
        return tc::make_tmap_u8(m, c.k, 2, dims, str, box, swizzle);
    };
    if (!map(&tmC, 128, PG, CU_TENSOR_MAP_SWIZZLE_128B) || !map(&tmCr, 64, PG, CU_TENSOR_MAP_SWIZZLE_64B) ||
        !map(&cut.rows8, 128, 8, CU_TENSOR_MAP_SWIZZLE_128B) || !map(&cut.row1, 128, 1, CU_TENSOR_MAP_SWIZZLE_128B))
        return GQLA_ERR_CUDA;
    tc::Fp8PairParams p{};
    p.B = c.B; p.S = S; p.s_q = c.s_q; p.h_q = d.h_q; p.rows_total = (int32_t)rows_total; p.row_blocks = (int32_t)row_blocks;
    p.balanced = balanced ? 1 : 0; p.W = workers; p.slack = whole_slack(d, c.s_q, true);
    p.n_rows = (int32_t)c.n_rows; p.n_pages = (int32_t)(c.n_rows / c.page_size);
    p.scale_log2 = c.scale * 1.4426950408889634f;
    p.q = (const __nv_bfloat16*)c.q; p.page_scale = c.k_scale;
    p.rows = RowMap{nullptr, c.block_table, c.max_pages, c.page_size};
    p.seqlens = c.seqlens; p.o_part = c.o_part; p.lse_part = c.lse_part; p.status = c.status;
    auto kern = tc::decode_fp8_pair_kernel<PG>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, tc::Fp8PairSmem::kTotal) != cudaSuccess) return GQLA_ERR_CUDA;
    return tc::launch_pdl(kern, dim3((unsigned)(2 * pairs)), dim3(tc::Fp8PairSmem::kThreads), tc::Fp8PairSmem::kTotal, st, p, tmC, tmCr,
                          cut) == cudaSuccess
               ? GQLA_OK
               : GQLA_ERR_CUDA;
}

template <int PG>
gqla_status tc_decode_fp8_paged(const Fp8PagedCall& c, cudaStream_t st) {
    if (on_pairs(*c.d, c.s_q, c.latent) && !few_pieces(c)) return tc_decode_fp8_pairs<PG>(c, st);
    const gqla_dims& d = *c.d;
    const int g = c.latent ? 1 : d.g, heads = d.h_q / g;
    const RowBlocks rb = row_blocks(c.s_q, heads);
    const int32_t plan_workers = c.S < 0 ? workers_of(d, c.s_q, c.latent) : 0;
    const int32_t workers = plan_workers > 0 ? token_workers(d, c.s_q, c.latent) : 0;
    const bool balanced = workers > 0;
    const int32_t S = c.S < 0 ? -c.S : c.S;
    const int64_t units = (balanced ? (int64_t)workers : (int64_t)c.B * S) * g * rb.count();
    if (units > 0x7fffffffLL) return GQLA_ERR_UNSUPPORTED;
    CUtensorMap tmK, tmR, tmV;
    tc::CutMaps<PG> cut;
    // the plane whose rows are values: the latent rows, or V
    const uint64_t vdims[3] = {c.latent ? (uint64_t)(d.r_kv + d.d_r) : (uint64_t)d.d_h, c.latent ? (uint64_t)c.n_rows : (uint64_t)d.g,
                               (uint64_t)c.n_rows};
    const uint64_t vstr[2] = {c.latent ? (uint64_t)c.k_stride : (uint64_t)d.d_h, (uint64_t)d.g * d.d_h};
    const int rank = c.latent ? 2 : 3;
    auto rows_map = [&](CUtensorMap* m, const uint8_t* base, uint32_t box_rows) {
        const uint32_t box[3] = {128, c.latent ? box_rows : 1u, box_rows};
        return tc::make_tmap_u8(m, base, rank, vdims, vstr, box, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    const uint8_t* values = c.latent ? c.k : c.v;
    if (!rows_map(&tmK, c.k, PG) || !rows_map(&tmV, values, PG) || !rows_map(&cut.rows8, values, 8) || !rows_map(&cut.row1, values, 1))
        return GQLA_ERR_CUDA;
    {
        const uint64_t dims[2] = {c.latent ? (uint64_t)(d.r_kv + d.d_r) : (uint64_t)d.d_r, (uint64_t)c.n_rows};
        const uint64_t str[1] = {(uint64_t)(c.latent ? c.k_stride : c.k_r_stride)};
        const uint32_t box[2] = {64, PG};
        if (!tc::make_tmap_u8(&tmR, c.latent ? c.k : c.k_r, 2, dims, str, box, CU_TENSOR_MAP_SWIZZLE_64B)) return GQLA_ERR_CUDA;
    }
    tc::Fp8PagedParams p{};
    p.B = c.B; p.S = S; p.s_q = c.s_q; p.h_q = d.h_q; p.g = g; p.hpg = heads;
    p.hb = rb.hb; p.n_hb = rb.n_hb; p.row_blocks = (int32_t)rb.count();
    while ((1 << p.hshift) < rb.hb) ++p.hshift;
    p.balanced = balanced ? 1 : 0; p.W = workers; p.plan_W = plan_workers; p.slack = whole_slack(d, c.s_q, c.latent);
    p.n_rows = (int32_t)c.n_rows; p.n_pages = (int32_t)(c.n_rows / c.page_size);
    p.scale_log2 = c.scale * 1.4426950408889634f;
    p.q = (const __nv_bfloat16*)c.q;
    p.k_scale = c.k_scale; p.r_scale = c.r_scale; p.v_scale = c.v_scale;
    p.cache = c.k;
    p.l2_stride = c.latent && c.k_stride <= 640 ? (int32_t)c.k_stride : 0;
    p.rows = RowMap{nullptr, c.block_table, c.max_pages, c.page_size};
    p.seqlens = c.seqlens; p.o_part = c.o_part; p.lse_part = c.lse_part; p.status = c.status;
    cudaError_t e;
    if (c.latent)
        e = rb.R == 16 ? launch_tc<16, true, PG>(p, tmK, tmR, tmV, cut, (unsigned)units, st)
                       : launch_tc<32, true, PG>(p, tmK, tmR, tmV, cut, (unsigned)units, st);
    else
        e = rb.R == 16 ? launch_tc<16, false, PG>(p, tmK, tmR, tmV, cut, (unsigned)units, st)
                       : launch_tc<32, false, PG>(p, tmK, tmR, tmV, cut, (unsigned)units, st);
    return e == cudaSuccess ? GQLA_OK : GQLA_ERR_CUDA;
}

gqla_status decode_fp8_paged(const Fp8PagedCall& c, void* out, float* lse, void* stream) {
    const gqla_dims* d = c.d;
    gqla_status s = check_dims(d);
    if (s != GQLA_OK) return s;
    if (c.dtype != GQLA_BF16 && c.dtype != GQLA_F32) return GQLA_ERR_DTYPE;
    if (c.B < 0 || c.s_q < 1 || c.S == 0 || c.S == -1 || c.S < -0x7fffffff || c.page_size < 1 || c.max_pages < 1 || c.n_rows < 0 || c.n_rows > 0x7fffffffLL)
        return GQLA_ERR_SHAPE;
    if (c.B == 0) return GQLA_OK;
    const bool rope = !c.latent && d->d_r > 0;
    if (c.q == nullptr || c.k == nullptr || c.k_scale == nullptr || c.block_table == nullptr || c.seqlens == nullptr || c.o_part == nullptr ||
        c.lse_part == nullptr || (!c.latent && (c.v == nullptr || c.v_scale == nullptr)) || (rope && (c.k_r == nullptr || c.r_scale == nullptr)))
        return GQLA_ERR_NULL;
    if (out == nullptr && lse != nullptr) return GQLA_ERR_NULL;
    if (!aligned(c.q, 16) || !aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.k_r, 16) || !aligned(c.o_part, 16) || !aligned(out, 16))
        return GQLA_ERR_ALIGN;
    const int32_t dv = c.latent ? d->r_kv : d->d_h;
    if ((c.latent && c.k_stride < d->r_kv + d->d_r) || (rope && c.k_r_stride < d->d_r)) return GQLA_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)stream;
    const int32_t S = c.S < 0 ? -c.S : c.S;
    s = GQLA_ERR_UNSUPPORTED;
    if (covers(*d, c.dtype, c.s_q, c.page_size, c.latent) && c.n_rows >= 1 && (c.latent ? c.k_stride : c.k_r_stride) % 16 == 0)
        s = c.page_size % 64 == 0   ? tc_decode_fp8_paged<64>(c, st)
            : c.page_size % 32 == 0 ? tc_decode_fp8_paged<32>(c, st)
                                    : tc_decode_fp8_paged<16>(c, st);
    if (s == GQLA_ERR_UNSUPPORTED) {
        if (dv > 32 * kGenericCols) return GQLA_ERR_UNSUPPORTED;
        Fp8PagedGeneric a{};
        a.q = c.q;
        a.kA = (const e4m3*)c.k; a.kB = (const e4m3*)c.k_r; a.v = (const e4m3*)(c.latent ? c.k : c.v);
        a.kv_heads = c.latent ? 1 : d->g;
        a.dA = c.latent ? d->r_kv + d->d_r : d->d_h; a.dB = rope ? d->d_r : 0; a.dv = dv;
        a.kA_stride = c.latent ? c.k_stride : (int64_t)d->g * d->d_h; a.kB_stride = c.k_r_stride;
        a.v_stride = a.kA_stride;
        a.sA = c.k_scale; a.sB = c.r_scale; a.sV = c.latent ? c.k_scale : c.v_scale;
        a.rows = RowMap{nullptr, c.block_table, c.max_pages, c.page_size};
        a.n_pages = (int32_t)(c.n_rows / c.page_size);
        a.seqlens = c.seqlens; a.B = c.B; a.S = S; a.s_q = c.s_q; a.h_q = d->h_q;
        a.scale = c.scale; a.o_part = c.o_part; a.lse_part = c.lse_part; a.status = c.status;
        const int64_t blocks = ((int64_t)c.B * S * c.s_q * d->h_q + 3) / 4;
        if (blocks > 0x7fffffffLL) return GQLA_ERR_SHAPE;
        if (c.dtype == GQLA_BF16) decode_fp8_paged_generic_kernel<__nv_bfloat16><<<(unsigned)blocks, 128, 0, st>>>(a);
        else decode_fp8_paged_generic_kernel<float><<<(unsigned)blocks, 128, 0, st>>>(a);
        s = cudaGetLastError() == cudaSuccess ? GQLA_OK : GQLA_ERR_CUDA;
    }
    if (s != GQLA_OK || out == nullptr) return s;
    return gqla_combine_splits(c.B, c.s_q * d->h_q, S, dv, c.dtype, c.o_part, c.lse_part, out, lse, stream);
}

}  // namespace

extern "C" {

gqla_status gqla_append_rope(const gqla_dims* d, gqla_dtype dtype, int32_t B, int64_t n_new, const int32_t* new_start,
                             const int32_t* seqlens, const void* c, int64_t c_row_stride, const void* k_r, int64_t k_r_row_stride,
                             const float* rope, int32_t rope_rows, gqla_rope_style style, const void* q_r, int64_t q_row_stride,
                             int64_t q_head_stride, void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride, void* cache,
                             int64_t cache_row_stride, int64_t cache_rows, const int64_t* seq_start, const int32_t* block_table,
                             int32_t max_pages, int32_t page_size, int32_t* status_word, void* stream) {
    const AppendCall call{dtype, B, n_new, new_start, seqlens, k_r, k_r_row_stride, rope, rope_rows, style, q_r, q_row_stride,
                          q_head_stride, q_out, q_out_row_stride, q_out_head_stride};
    const gqla_status s = check_append(d, call);
    if (s != GQLA_OK) return s;
    if (block_table != nullptr && (max_pages < 1 || page_size < 1)) return GQLA_ERR_SHAPE;
    if (B == 0 || n_new == 0) return GQLA_OK;
    if (c == nullptr || cache == nullptr || (block_table == nullptr) == (seq_start == nullptr)) return GQLA_ERR_NULL;
    if (c_row_stride < d->r_kv || cache_row_stride < d->r_kv + d->d_r || cache_rows < 0) return GQLA_ERR_SHAPE;
    const bool vec = vectors(*d, call) && d->r_kv % 8 == 0 && c_row_stride % 8 == 0 && cache_row_stride % 8 == 0 && aligned(c, 16) &&
                     aligned(cache, 16);
    AppendArgs a{};
    fill(a, *d, call);
    a.c = c; a.c_stride = c_row_stride; a.r_kv = d->r_kv;
    a.items = ItemsOfRow(!vec ? d->r_kv : dtype == GQLA_BF16 ? d->r_kv / 8 : d->r_kv / 4);
    a.cache = cache; a.cache_stride = cache_row_stride; a.cache_rows = cache_rows;
    a.rows = block_table != nullptr ? RowMap{nullptr, block_table, max_pages, page_size} : RowMap{seq_start, nullptr, 0, 1};
    a.status = status_word;
    // a row per warp while that does not fill the GPU, four beyond (each lane then keeps eight loads of a latent part of 1 KB in
    // flight).  One and four rows a warp, in a graph: 4000 rows 4.7 and 5.4 us, 6000 6.9 and 4.8, 8192 8.3 and 7.1, 12000 11.4 and 8.0, 16000
    // 15.6 and 9.0 (eight: 12000 8.3, 39000 20.3 against 19.8 with four, 98000 40.9 against 41.3)
    a.per_warp = n_new >= 8192 ? kAppendMostRows : 1;
    const int64_t rows_per_block = (int64_t)a.per_warp * (kAppendThreads / 32);
    const int64_t kv = (n_new + rows_per_block - 1) / rows_per_block;
    a.kv_blocks = (int32_t)kv;
    const int64_t blocks = kv + query_blocks(*d, call, vec, kAppendThreads);
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == GQLA_BF16)
        return launch_append(vec ? append_rope_kernel<__nv_bfloat16, true> : append_rope_kernel<__nv_bfloat16, false>, a, blocks,
                             kAppendThreads, st);
    return launch_append(vec ? append_rope_kernel<float, true> : append_rope_kernel<float, false>, a, blocks, kAppendThreads, st);
}

gqla_status gqla_append_rope_fp8(const gqla_dims* d, gqla_dtype dtype, int32_t B, int64_t n_new, const int32_t* new_start,
                                 const int32_t* seqlens, const void* c, int64_t c_row_stride, const void* k_r, int64_t k_r_row_stride,
                                 const float* rope, int32_t rope_rows, gqla_rope_style style, const void* q_r, int64_t q_row_stride,
                                 int64_t q_head_stride, void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                 uint8_t* cache8, int64_t cache_row_stride, int64_t cache_rows, float* page_scale,
                                 const int32_t* block_table, int32_t max_pages, int32_t page_size, int32_t* status_word,
                                 void* stream) {
    const AppendCall call{dtype, B, n_new, new_start, seqlens, k_r, k_r_row_stride, rope, rope_rows, style, q_r, q_row_stride,
                          q_head_stride, q_out, q_out_row_stride, q_out_head_stride};
    const gqla_status s = check_append(d, call);
    if (s != GQLA_OK) return s;
    if (max_pages < 1 || page_size < 1) return GQLA_ERR_SHAPE;
    if (B == 0 || n_new == 0) return GQLA_OK;
    if (c == nullptr || cache8 == nullptr || page_scale == nullptr || block_table == nullptr) return GQLA_ERR_NULL;
    if (c_row_stride < d->r_kv || cache_row_stride < d->r_kv + d->d_r || cache_rows < 0 || cache_rows > 0x7fffffffLL)
        return GQLA_ERR_SHAPE;
    AppendFp8Args a{};
    a.plane[0] = Fp8Plane{c, c_row_stride, 1, d->r_kv, d->d_r > 0, cache8, cache_row_stride, page_scale, 1};
    const bool vec = vectors(*d, call) && d->r_kv % 8 == 0 && c_row_stride % 8 == 0 && cache_row_stride % 8 == 0 && aligned(c, 16) &&
                     aligned(cache8, 8);
    return launch_append_fp8(*d, call, a, vec, block_table, max_pages, page_size, cache_rows, status_word, (cudaStream_t)stream);
}

gqla_status gqla_append_planes_fp8(const gqla_dims* d, gqla_dtype dtype, int32_t B, int64_t n_new, const int32_t* new_start,
                                   const int32_t* seqlens, const void* k_c, const void* v, const void* k_r, int64_t k_r_row_stride,
                                   const float* rope, int32_t rope_rows, gqla_rope_style style, const void* q_r, int64_t q_row_stride,
                                   int64_t q_head_stride, void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride,
                                   uint8_t* k_c8, uint8_t* v8, uint8_t* k_r8, int64_t k_r8_row_stride, int64_t n_rows,
                                   float* k_scale, float* v_scale, float* r_scale, const int32_t* block_table, int32_t max_pages,
                                   int32_t page_size, int32_t* status_word, void* stream) {
    const AppendCall call{dtype, B, n_new, new_start, seqlens, k_r, k_r_row_stride, rope, rope_rows, style, q_r, q_row_stride,
                          q_head_stride, q_out, q_out_row_stride, q_out_head_stride};
    const gqla_status s = check_append(d, call);
    if (s != GQLA_OK) return s;
    if (max_pages < 1 || page_size < 1) return GQLA_ERR_SHAPE;
    if (B == 0 || n_new == 0) return GQLA_OK;
    if (k_c == nullptr || v == nullptr || k_c8 == nullptr || v8 == nullptr || k_scale == nullptr || v_scale == nullptr ||
        block_table == nullptr || (d->d_r > 0 && (k_r8 == nullptr || r_scale == nullptr)))
        return GQLA_ERR_NULL;
    if ((d->d_r > 0 && k_r8_row_stride < d->d_r) || n_rows < 0 || n_rows > 0x7fffffffLL) return GQLA_ERR_SHAPE;
    const int64_t stride = (int64_t)d->g * d->d_h;
    AppendFp8Args a{};
    a.plane[0] = Fp8Plane{k_c, stride, d->g, d->d_h, 0, k_c8, stride, k_scale, d->g};
    a.plane[1] = Fp8Plane{v, stride, d->g, d->d_h, 0, v8, stride, v_scale, d->g};
    if (d->d_r > 0) a.plane[2] = Fp8Plane{nullptr, 0, 1, 0, 1, k_r8, k_r8_row_stride, r_scale, 1};
    const bool vec = vectors(*d, call) && d->d_h % 8 == 0 && k_r8_row_stride % 8 == 0 && aligned(k_c, 16) && aligned(v, 16) &&
                     aligned(k_c8, 8) && aligned(v8, 8) && aligned(k_r8, 8);
    return launch_append_fp8(*d, call, a, vec, block_table, max_pages, page_size, n_rows, status_word, (cudaStream_t)stream);
}

gqla_status gqla_decode_absorb_fp8_paged(const gqla_dims* d, gqla_dtype dtype, int32_t B, int32_t s_q, float scale, int32_t num_splits,
                                         const void* q_hat, const uint8_t* cache8, int64_t cache_row_stride, int64_t cache_rows,
                                         const float* page_scale, const int32_t* block_table, int32_t max_pages, int32_t page_size,
                                         const int32_t* seqlens, float* o_part, float* lse_part, void* out, float* lse,
                                         int32_t* status_word, void* stream) {
    return decode_fp8_paged({d, dtype, B, s_q, scale, num_splits, q_hat, cache8, nullptr, nullptr, cache_row_stride, 0, cache_rows,
                             page_scale, nullptr, nullptr, block_table, max_pages, page_size, seqlens, o_part, lse_part, status_word,
                             true}, out, lse, stream);
}

gqla_status gqla_decode_gqa_fp8_paged(const gqla_dims* d, gqla_dtype dtype, int32_t B, int32_t s_q, float scale, int32_t num_splits,
                                      const void* q, const uint8_t* k_c8, const uint8_t* v8, const uint8_t* k_r8,
                                      int64_t k_r8_row_stride, int64_t n_rows, const float* k_scale, const float* v_scale,
                                      const float* r_scale, const int32_t* block_table, int32_t max_pages, int32_t page_size,
                                      const int32_t* seqlens, float* o_part, float* lse_part, void* out, float* lse,
                                      int32_t* status_word, void* stream) {
    return decode_fp8_paged({d, dtype, B, s_q, scale, num_splits, q, k_c8, v8, k_r8, 0, k_r8_row_stride, n_rows, k_scale, v_scale,
                             r_scale, block_table, max_pages, page_size, seqlens, o_part, lse_part, status_word, false}, out, lse,
                            stream);
}

int32_t gqla_fp8_paged_workers(const gqla_dims* d, gqla_dtype dtype, int32_t s_q, int32_t page_size, int32_t path) {
    if (check_dims(d) != GQLA_OK || s_q < 1 || page_size < 1) return -1;
    return covers(*d, dtype, s_q, page_size, path == 0) ? workers_of(*d, s_q, path == 0) : 0;
}

}  // extern "C"
