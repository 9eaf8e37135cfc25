// Appending a step's or a prompt's rows to the KV cache with the position rotation applied on the way (the decoupled-RoPE
// key k^R of Sec. 3.1 enters the cache rotated; the paper takes the rotation as done).  Three forms:
//
//   latent rows   [c ; R_t k_r] in the storage type, packed or paged cache                     append_rope_kernel
//   E4M3 pages    the same row as codes with one scale per page, or the planes K_C, V, k_R
//                 with a scale per page and group (k_R: per page)                              append_fp8_kernel
//
// and in each the step's queries q_r are rotated by the same launch.  R_t turns the pair (a, b) by the angle whose cosine and
// sine row t of the caller's table holds: (a cos - b sin, a sin + b cos) in fp32, rounded once to what is stored.
//
// A page's scale is a power of two, s = max over the page's rows so far of the smallest 2^e with |x| <= 448 * 2^e (e >= -40).  A
// later row may raise it; the page's older codes are then coded anew, which shifts their exponents and loses nothing but what
// falls below 2^-9 of the new scale.  With a power of two the products by 1 / s are exact: a code is the value rounded once.
//
// What bounds them: HBM on prompts (rows are read once and written once), the chain start -> length -> block table -> row
// on a step.
#pragma once
#include <float.h>

#include "common.cuh"
#include "tc_common.cuh"

namespace gqla {

constexpr int32_t kStatusShape = 2;  // == GQLA_ERR_SHAPE: a position behind the rotation table or the block table, a page outside the cache
constexpr int kAppendThreads = 256;
constexpr int kSmallestScaleExp = -40;

struct NewRows {
    int32_t B;
    int64_t n;               // rows in all
    const int32_t* start;    // [B + 1]: sequence b's new rows are [start[b], start[b + 1])
    const int32_t* seqlens;  // [B], the new rows counted
    // Sequence that owns new row i (a row behind all of them: the last).
    __device__ __forceinline__ int32_t seq_of(int32_t i) const {
        int32_t lo = 0, hi = B - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (start[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
    // The row's position in that sequence; negative where the row is skipped: in front of the sequence, or behind the last one's rows.
    __device__ __forceinline__ int32_t pos_of(int32_t i, int32_t b) const {
        const int32_t end = start[b + 1], T = seqlens[b];  // (both loads at once: a step waits for them)
        return i < end ? T - (end - i) : -1;
    }
};

// Largest b in [0, B) with at(b) <= x, at ascending, at(0) <= x: a load per lane and round, 32-fold per round (a bisection is a chain of
// loads, which is what a step's append waits for).  All lanes of the warp call it.
template <typename F>
__device__ __forceinline__ int32_t warp_last(int32_t B, int32_t x, F at) {
    const int lane = threadIdx.x & 31;
    int32_t lo = 0, size = B;
    while (size > 1) {
        const int32_t step = (size + 31) >> 5, i = lane * step;
        const int32_t c = __popc(__ballot_sync(0xffffffffu, i < size && at(lo + (i < size ? i : 0)) <= x));
        const int32_t skip = (c > 0 ? c - 1 : 0) * step;
        lo += skip;
        size = size - skip < step ? size - skip : step;
    }
    return lo;
}

struct RopeTable {
    const float* cs;  // [rows, d_r]: cosines in the first half of a row, sines in the second
    int32_t rows, d_r, halves;  // halves: pairs (i, i + d_r / 2), otherwise (2 i, 2 i + 1)
};

struct QueryRows {  // [n, h_q, d_r], the last dimension contiguous; src null: none
    const void* src;
    void* dst;
    int64_t src_tok, src_head, dst_tok, dst_head;
    int32_t h_q;
};

__device__ __forceinline__ void append_error(int32_t* status, int32_t where) {
    if (status != nullptr) atomicCAS(status, 0, kStatusShape | (where << 8));
}

// Eight elements as floats (16-byte aligned for bf16, 32 bytes of fp32 as two loads).
__device__ __forceinline__ void unpack8(const uint4& u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* v) { unpack8(*reinterpret_cast<const uint4*>(p), v); }
__device__ __forceinline__ void load8(const float* p, float* v) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v) {
    *reinterpret_cast<uint4*>(p) = make_uint4(tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]), tc::pack_bf16(v[4], v[5]),
                                              tc::pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float* v) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(e4m3* p, const float* v) {
    *reinterpret_cast<uint2*>(p) =
        make_uint2((uint32_t)float2_to_e4m3x2(v[0], v[1]) | ((uint32_t)float2_to_e4m3x2(v[2], v[3]) << 16),
                   (uint32_t)float2_to_e4m3x2(v[4], v[5]) | ((uint32_t)float2_to_e4m3x2(v[6], v[7]) << 16));
}
__device__ __forceinline__ void stf(e4m3* p, float v) { p->code = (uint8_t)(float2_to_e4m3x2(v, 0.f) & 0xff); }

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float x = a;
    a = fmaf(x, c, -b * s);
    b = fmaf(x, s, b * c);
}

// N = 4 or 8 of them.
template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, float* v) {
    if constexpr (N == 8) {
        load8(p, v);
    } else if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
        v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
    }
}
__device__ __forceinline__ void store4(e4m3* p, const float* v) {
    *reinterpret_cast<uint32_t*>(p) = (uint32_t)float2_to_e4m3x2(v[0], v[1]) | ((uint32_t)float2_to_e4m3x2(v[2], v[3]) << 16);
}

// A rotation item: 2 N elements, item i of d_r / (2 N): N each from 2 N i and 2 N i + N on, or from N i and N i + d_r / 2 with halves.
// N = 8 and 4 are vectors (4: half the registers, for pages), N = 1 a pair.
template <int N>
struct RopeItem {
    static constexpr int kN = N;
    static __host__ __device__ int count(int d_r) { return d_r / (2 * N); }
    float a[kN], b[kN];
    int ca, cb;  // first columns of the parts
    __device__ __forceinline__ RopeItem(const RopeTable& t, int i)
        : ca(t.halves ? i * kN : 2 * i * kN), cb(t.halves ? i * kN + t.d_r / 2 : (2 * i + 1) * kN) {}
    template <typename T>
    __device__ __forceinline__ void load(const T* x) {
        if constexpr (N > 1) {
            load_n<N>(x + ca, a);
            load_n<N>(x + cb, b);
        } else {
            a[0] = ldf(x + ca);
            b[0] = ldf(x + cb);
        }
    }
    __device__ __forceinline__ void rotate(const RopeTable& t, int32_t pos) {
        const float* cs = t.cs + (int64_t)pos * t.d_r;
        const int half = t.d_r / 2;
        const int f = t.halves ? ca : ca / 2;
        if constexpr (N > 1) {
            float c[N], s[N];
            load_n<N>(cs + f, c);
            load_n<N>(cs + half + f, s);
            if (t.halves) {
#pragma unroll
                for (int k = 0; k < N; ++k) turn(a[k], b[k], c[k], s[k]);
            } else {  // pairs within each part: N frequencies over both
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    turn(a[2 * k], a[2 * k + 1], c[k], s[k]);
                    turn(b[2 * k], b[2 * k + 1], c[N / 2 + k], s[N / 2 + k]);
                }
            }
        } else {
            turn(a[0], b[0], cs[f], cs[half + f]);
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* y) const {
        if constexpr (N == 8) {
            store8(y + ca, a);
            store8(y + cb, b);
        } else if constexpr (N == 4) {
            store4(y + ca, a);
            store4(y + cb, b);
        } else {
            stf(y + ca, a[0]);
            stf(y + cb, b[0]);
        }
    }
};

// The queries' share of a launch: item index `i` counts (row, head, rotation item).
template <typename T, bool VEC>
__device__ __forceinline__ void rotate_queries(const NewRows& nr, const RopeTable& rope, const QueryRows& q, int64_t i, int32_t* status) {
    const int per = RopeItem<VEC ? 8 : 1>::count(rope.d_r);
    if (i >= nr.n * q.h_q * per) return;
    const int item = (int)(i % per), head = (int)(i / per % q.h_q);
    const int32_t tok = (int32_t)(i / per / q.h_q);
    const int32_t b = nr.seq_of(tok), pos = nr.pos_of(tok, b);
    if (pos < 0) return;
    if (pos >= rope.rows) return append_error(status, 1);
    RopeItem<VEC ? 8 : 1> x(rope, item);
    x.load((const T*)q.src + tok * q.src_tok + head * q.src_head);
    x.rotate(rope, pos);
    x.store((T*)q.dst + tok * q.dst_tok + head * q.dst_head);
}

// Where row `pos` of sequence b goes; negative where the block table or the page number does not allow it.
__device__ __forceinline__ int64_t checked_row(const RowMap& rows, int32_t b, int32_t pos, int64_t n_rows, int32_t* status) {
    int64_t row;
    if (rows.paged()) {
        const int32_t k = pos / rows.page_size;
        const int32_t page = k < rows.max_pages ? rows.block_table[(int64_t)b * rows.max_pages + k] : -1;
        row = page < 0 ? -1 : (int64_t)page * rows.page_size + pos % rows.page_size;
    } else {
        row = rows.seq_start[b] + pos;
    }
    if (row >= 0 && row < n_rows) return row;
    append_error(status, 2);
    return -1;
}

// i / per for 0 <= i < 2^10 by a multiplication with m = ceil(2^32 / per): exact while i (m per - 2^32) < 2^32, which holds for
// per < 2^22, and i < per beyond.
struct ItemsOfRow {
    int32_t per;
    uint32_t recip;  // m; 0: per is 1
    ItemsOfRow() = default;
    explicit ItemsOfRow(int32_t per_) : per(per_), recip(per_ > 1 ? (uint32_t)(((1ull << 32) + (uint32_t)per_ - 1) / (uint32_t)per_) : 0u) {}
    __device__ __forceinline__ int quotient(int i) const { return recip != 0 ? (int)__umulhi((uint32_t)i, recip) : i; }
};

struct AppendArgs {
    NewRows nr;
    RopeTable rope;
    QueryRows q;
    const void *c, *k_r;
    int64_t c_stride, k_r_stride;
    int32_t r_kv;
    void* cache;
    int64_t cache_stride, cache_rows;
    RowMap rows;
    int32_t per_warp, kv_blocks;  // new rows of a warp; blocks behind kv_blocks rotate queries
    ItemsOfRow items;             // vectors or elements of a latent part
    int32_t* status;
};

constexpr int kAppendMostRows = 4;  // new rows of a warp

// Item i, i + step, i + 2 step, .. of rows of `per` items each, without a division per item.
struct RowItems {
    int row, col, row_step, col_step, per;
    __device__ __forceinline__ RowItems(int i, int step, const ItemsOfRow& of)
        : row(of.quotient(i)), col(i - row * of.per), row_step(of.quotient(step)), col_step(step - row_step * of.per), per(of.per) {}
    __device__ __forceinline__ void next() {
        row += row_step;
        col += col_step;
        if (col >= per) {
            col -= per;
            ++row;
        }
    }
};

// A warp takes per_warp new rows: their places are looked up by a lane each, the latent parts copied eight 16-byte vectors a lane
// at a time (49000 rows of 1152 bytes: 26.5 us, 5.2 TB/s; 41.7 with a block per sixteen rows and one vector a thread in flight), the RoPE parts rotated an
// item a lane.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kAppendThreads) append_rope_kernel(const AppendArgs a) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if ((int)blockIdx.x >= a.kv_blocks)
        return rotate_queries<T, VEC>(a.nr, a.rope, a.q, (int64_t)(blockIdx.x - a.kv_blocks) * kAppendThreads + threadIdx.x, a.status);
    const int lane = threadIdx.x & 31;
    const int64_t tok0 = ((int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5)) * a.per_warp;
    if (tok0 >= a.nr.n) return;
    const int n = (int)(a.nr.n - tok0 < a.per_warp ? a.nr.n - tok0 : a.per_warp);
    constexpr int kAhead = 8;
    RowItems it(lane, 32, a.items);
    uint4 v[kAhead];
    auto fetch = [&](RowItems from) {
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
            if (from.row < n) v[h] = reinterpret_cast<const uint4*>((const T*)a.c + (tok0 + from.row) * a.c_stride)[from.col];
            from.next();
        }
    };
    if constexpr (VEC) fetch(it);  // (before the rows' places are known)
    int64_t my_row = -1;
    int32_t my_pos = 0;
    if (lane < n) {
        const int32_t tok = (int32_t)tok0 + lane, b = a.nr.seq_of(tok);
        my_pos = a.nr.pos_of(tok, b);
        if (my_pos >= a.rope.rows && a.rope.d_r > 0) append_error(a.status, 1);
        else if (my_pos >= 0) my_row = checked_row(a.rows, b, my_pos, a.cache_rows, a.status);
    }
    auto row_of = [&](int k) { return __shfl_sync(0xffffffffu, my_row, k < n ? k : 0); };
    if constexpr (VEC) {
        for (int i0 = 0; i0 < n * it.per; i0 += 32 * kAhead) {
            if (i0 > 0) fetch(it);
#pragma unroll
            for (int h = 0; h < kAhead; ++h) {
                const int64_t row = row_of(it.row);
                if (it.row < n && row >= 0) reinterpret_cast<uint4*>((T*)a.cache + row * a.cache_stride)[it.col] = v[h];
                it.next();
            }
        }
    } else {
        for (int i0 = 0; i0 < n * it.per; i0 += 32) {
            const int64_t row = row_of(it.row);
            if (it.row < n && row >= 0)
                ((T*)a.cache + row * a.cache_stride)[it.col] = ((const T*)a.c + (tok0 + it.row) * a.c_stride)[it.col];
            it.next();
        }
    }
    const int turns = RopeItem<VEC ? 8 : 1>::count(a.rope.d_r);
    for (int i0 = 0; i0 < n * turns; i0 += 32) {
        const int i = i0 + lane, k = turns > 0 ? i / turns : 0;
        const int64_t row = row_of(k);
        const int32_t pos = __shfl_sync(0xffffffffu, my_pos, k < n ? k : 0);
        if (k >= n || row < 0) continue;
        RopeItem<VEC ? 8 : 1> x(a.rope, i % turns);
        x.load((const T*)a.k_r + (tok0 + k) * a.k_r_stride);
        x.rotate(a.rope, pos);
        x.store((T*)a.cache + row * a.cache_stride + a.r_kv);
    }
}

// ------------------------------------------------------------------------------------------------ E4M3 pages

// Smallest 2^e with amax <= 448 * 2^e, e >= least (finite amax >= 0): amax = (1 + f) 2^x and 448 = 1.75 * 2^8.
__device__ __forceinline__ float pow2_scale(float amax, int least) {
    const uint32_t bits = __float_as_uint(amax);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
    if (e < least) e = least;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
// Largest magnitude of bf16 values, a running maximum in each half of `m` (signs of no meaning).  A NaN beside a number is passed over.
__device__ __forceinline__ uint32_t bf16_max(uint32_t m, const uint4& u) {
    auto max2 = [](uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    };
    return max2(m, max2(max2(u.x, u.y), max2(u.z, u.w)));
}
// The largest finite magnitude, from that maximum: where it is an infinity, `each` hands all chunks again.
template <typename F>
__device__ __forceinline__ float bf16_finite_max(uint32_t m, F each) {
    m &= 0x7fff7fffu;
    if (__vcmpgeu2(m, 0x7f807f80u) != 0) {
        m = 0;
        each([&](const uint4& u) {
            const uint32_t w[4] = {u.x & 0x7fff7fffu, u.y & 0x7fff7fffu, u.z & 0x7fff7fffu, u.w & 0x7fff7fffu};
            for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & __vcmpltu2(w[i], 0x7f807f80u));
        });
    }
    return __uint_as_float(max(m & 0xffffu, m >> 16) << 16);
}
__device__ __forceinline__ float finite_max(float m, float x) {
    const float a = fabsf(x);
    return a <= FLT_MAX && a > m ? a : m;
}

struct Fp8Plane {
    const void* a;     // first part of a row: width elements, copied
    int64_t a_stride;  // between the rows of the source
    int32_t a_heads, a_width;
    int32_t rope_heads;  // 1: a rotated part of d_r elements from k_r follows (or is all there is, with a_width == 0)
    uint8_t* dst;
    int64_t dst_stride;
    float* scale;  // [pages, heads]
    int32_t heads;
    ItemsOfRow copied, turned, coded;  // vectors or elements of the first part, rotation items, vectors or elements of a row of codes
};

struct AppendFp8Args {
    NewRows nr;
    RopeTable rope;
    QueryRows q;
    const void* k_r;
    int64_t k_r_stride;
    Fp8Plane plane[3];
    int32_t heads_in_all, n_pages;
    const int32_t* block_table;
    int32_t max_pages, page_size;
    int64_t kv_blocks;  // (unit, head) blocks; those behind rotate queries
    int32_t unit_shift;  // k of the units, -1: by rows
    int32_t held;        // chunks of a thread that its shared memory has room for
    int32_t* status;
};

// A block takes one head of one page that gets new rows.  Units of pages, without a prefix sum over the sequences:
//   by rows    unit u is new row u, if that is the first new one of its page (steps: fewer rows than the other bound)
//   otherwise  unit u of sequence b is its page number u - unit0(b) from the first touched one on, unit0(b) = (start[b] >> k) + 2 b
//              with 2^k <= page: n new rows touch at most (n - 1) / page + 2 pages, and successive unit0 are at least that far apart.
// What is left over exits.
// The first sixteen chunks of a thread stay in its shared memory between the maximum and the coding: all of a page of 64 latent rows
// with 256 threads, of 64 rows of one head of a plane with 64; larger pages read the rest again, from L1 or L2.  They come by
// asynchronous copies, which cost no registers while they are on their way.  Few warps of many chunks, since looking the unit up costs
// each warp some 400 instructions.  49000 latent rows and 20000 rows into the planes: 27.0 and 34.4 us in a graph (3.8 and 4.2 TB/s); twice
// the threads with eight chunks each 31.4 and 39.0, those chunks in registers 40.0 and 43.4.  Pages of 16, 32, 128 and 256 rows: 41.4, 28.4,
// 47.8 and 65.2 us, planes 60.9, 39.7, 48.5 and 74.6 -- small pages have a look-up for few rows, large ones read twice what is not held and
// have fewer blocks.  fp32 rows are not held either: 56.8 and 64.9.
constexpr int kLatentThreads = 256, kPlaneThreads = 64;
template <typename T, bool VEC, int THREADS>
struct HeldChunks {
    static constexpr int kPer = VEC && sizeof(T) == 2 ? 16 : 0;  // most of a thread
    static constexpr int kBytes = THREADS * 16;                 // of one each
};
template <typename T, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kLatentThreads ? 3 : 16) append_fp8_kernel(const AppendFp8Args a) {
    extern __shared__ uint4 append_held[];
    constexpr int kWarps = THREADS / 32;
    __shared__ float red[kWarps];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if ((int64_t)blockIdx.x >= a.kv_blocks)
        return rotate_queries<T, VEC>(a.nr, a.rope, a.q, ((int64_t)blockIdx.x - a.kv_blocks) * THREADS + threadIdx.x, a.status);
    const int32_t unit = THREADS == kLatentThreads ? (int32_t)blockIdx.x : (int32_t)(blockIdx.x / (unsigned)a.heads_in_all);
    int head = (int)(blockIdx.x - (unsigned)unit * (unsigned)a.heads_in_all);
    const int page = a.page_size;
    const int32_t b = a.unit_shift < 0 ? warp_last(a.nr.B, unit, [&](int32_t i) { return a.nr.start[i]; })
                                       : warp_last(a.nr.B, unit, [&](int32_t i) { return (a.nr.start[i] >> a.unit_shift) + 2 * i; });
    const int32_t s0 = a.nr.start[b], n = a.nr.start[b + 1] - s0;
    const int32_t T_len = a.nr.seqlens[b], first = T_len - n;
    if (n <= 0 || T_len <= 0) return;
    int32_t k;  // page of the sequence
    if (a.unit_shift < 0) {
        const int32_t pos = first + unit - s0;
        if (pos < 0 || pos >= T_len || (unit != s0 && pos % page != 0)) return;  // (T_len and on: rows behind the last sequence's)
        k = pos / page;
    } else {
        k = (first > 0 ? first / page : 0) + unit - ((s0 >> a.unit_shift) + 2 * b);
        if (k < 0 || (int64_t)k * page >= T_len) return;
    }
    const int32_t p0 = k * page;
    const int32_t lo = p0 > first ? p0 : first;  // new rows [lo, hi) of this page; first < p0 + page by the choice of k
    int32_t hi = T_len - p0 < page ? T_len : p0 + page;
    const int32_t pid = k < a.max_pages ? a.block_table[(int64_t)b * a.max_pages + k] : -1;  // (looked at behind the loads of the rows)
    if (a.rope.d_r > 0 && hi > a.rope.rows) {  // rows behind the rotation table are left out
        if (threadIdx.x == 0) append_error(a.status, 1);
        hi = a.rope.rows;
        if (hi <= lo) return;
    }
    int pl = 0;
    if constexpr (THREADS == kPlaneThreads) {  // (latent rows: one plane of one head, fields at fixed places)
        while (head >= a.plane[pl].heads) head -= a.plane[pl++].heads;
    } else {
        head = 0;
    }
    const Fp8Plane& P = a.plane[pl];
    const T* src = (const T*)P.a + (int64_t)(s0 + lo - first) * P.a_stride + head * P.a_width;
    const T* rsrc = (const T*)a.k_r + (int64_t)(s0 + lo - first) * a.k_r_stride;
    const int width = P.a_width + (P.rope_heads ? a.rope.d_r : 0);
    const int rows = hi - lo;
    const int tid = threadIdx.x;

    // largest finite magnitude of the new rows
    constexpr int kHeld = HeldChunks<T, VEC, THREADS>::kPer;
    constexpr int kElems = VEC ? 8 : 1;
    float amax = 0.f;
    const RowItems a0(tid, THREADS, P.copied);
    const int a_rows = P.a_width > 0 ? rows : 0;
    // Calls f(h, offset) for the held chunks, offset in elements for rows of `stride`; leaves `rest` at the first that is not held.
    RowItems rest = a0;
    auto each_held = [&](int64_t stride, auto f) {
        if (a0.col_step == 0) {  // one column per thread
            int64_t off = a0.row * stride + a0.col * 8;
            const int64_t step = a0.row_step * stride;
            int row = a0.row;
#pragma unroll 4
            for (int h = 0; h < a.held; ++h, row += a0.row_step, off += step)
                if (row < a_rows) f(h, off);
            rest.row = row;
        } else {
            rest = a0;
#pragma unroll 1
            for (int h = 0; h < a.held; ++h, rest.next())
                if (rest.row < a_rows) f(h, rest.row * stride + rest.col * 8);
        }
    };
    uint4* const held = append_held + tid;
    if constexpr (kHeld > 0) {
        each_held(P.a_stride, [&](int h, int64_t off) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(held + h * THREADS)), "l"(src + off) : "memory");
        });
    }
    const RowItems r0(tid, THREADS, P.turned);
    const int r_rows = P.rope_heads ? rows : 0;
    if (pid < 0 || pid >= a.n_pages) {
        if (tid == 0) append_error(a.status, 2);
        if constexpr (kHeld > 0) asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    e4m3* page_dst = (e4m3*)P.dst + (int64_t)pid * page * P.dst_stride + (int64_t)head * width;
    e4m3* dst = page_dst + (int64_t)(lo - p0) * P.dst_stride;
    float* const scale_at = P.scale + (int64_t)pid * P.heads + head;
    const float s_old = lo > p0 ? *scale_at : 0.f;  // the page's older rows, if it has any, hold it to this
    using Turn = RopeItem<VEC ? 4 : 1>;
    auto turned = [&](const RowItems& it) {
        Turn x(a.rope, it.col);
        x.load(rsrc + (int64_t)it.row * a.k_r_stride);
        x.rotate(a.rope, lo + it.row);
        return x;
    };
    auto turned_max = [&](const Turn& x) {
#pragma unroll
        for (int e = 0; e < Turn::kN; ++e) amax = finite_max(finite_max(amax, x.a[e]), x.b[e]);
    };
    // of latent rows the first two items stay in registers: all of a page of 64.  (In the planes one block of 2 g + 1 has any.)
    constexpr bool kHoldTurned = THREADS == kLatentThreads;
    RowItems r1 = r0;
    r1.next();
    RowItems r2 = r0;
    Turn t0(a.rope, r0.col), t1(a.rope, r1.col);
    if constexpr (kHoldTurned) {
        r2 = r1;
        r2.next();
        if (r0.row < r_rows) t0 = turned(r0);
        if (r1.row < r_rows) t1 = turned(r1);
        if (r0.row < r_rows) turned_max(t0);
        if (r1.row < r_rows) turned_max(t1);
    }
    for (RowItems it = r2; it.row < r_rows; it.next()) turned_max(turned(it));
    if constexpr (kHeld > 0) {
        asm volatile("cp.async.wait_all;" ::: "memory");  // (a thread reads back what it has copied itself)
        uint32_t top = 0;
        each_held(0, [&](int h, int64_t) { top = bf16_max(top, held[h * THREADS]); });
        amax = fmaxf(amax, bf16_finite_max(top, [&](auto f) { each_held(0, [&](int h, int64_t) { f(held[h * THREADS]); }); }));
    }
    for (RowItems it = rest; it.row < a_rows; it.next()) {
        const T* x = src + (int64_t)it.row * P.a_stride + it.col * kElems;
        if constexpr (VEC) {
            float v[8];
            load8(x, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = finite_max(amax, v[e]);
        } else {
            amax = finite_max(amax, ldf(x));
        }
    }
    amax = warp_max(amax);
    if ((tid & 31) == 0) red[tid >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) amax = fmaxf(amax, red[w]);
    const float need = pow2_scale(amax, kSmallestScaleExp);
    const float s = need > s_old ? need : s_old;
    const float inv = 1.f / s;

    if (lo > p0 && s > s_old) {  // the older rows under the larger scale
        const float ratio = s_old * inv;
        for (RowItems it(tid, THREADS, P.coded); it.row < lo - p0; it.next()) {
            e4m3* y = page_dst + (int64_t)it.row * P.dst_stride + it.col * kElems;
            if constexpr (VEC) {
                const uint2 u = *reinterpret_cast<const uint2*>(y);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e4m3_to_float((uint8_t)((e < 4 ? u.x : u.y) >> (8 * (e & 3)))) * ratio;
                store8(y, v);
            } else {
                stf(y, ldf(y) * ratio);
            }
        }
    }
    if constexpr (kHeld > 0) {
        each_held(P.dst_stride, [&](int h, int64_t off) {
            float v[8];
            unpack8(held[h * THREADS], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= inv;
            store8(dst + off, v);
        });
    }
    for (RowItems it = rest; it.row < a_rows; it.next()) {
        const T* x = src + (int64_t)it.row * P.a_stride + it.col * kElems;
        e4m3* y = dst + (int64_t)it.row * P.dst_stride + it.col * kElems;
        if constexpr (VEC) {
            float v[8];
            load8(x, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= inv;
            store8(y, v);
        } else {
            stf(y, ldf(x) * inv);
        }
    }
    auto store_turned = [&](Turn& x, int row) {
#pragma unroll
        for (int e = 0; e < Turn::kN; ++e) {
            x.a[e] *= inv;
            x.b[e] *= inv;
        }
        x.store(dst + (int64_t)row * P.dst_stride + P.a_width);
    };
    if constexpr (kHoldTurned) {
        if (r0.row < r_rows) store_turned(t0, r0.row);
        if (r1.row < r_rows) store_turned(t1, r1.row);
    }
    for (RowItems it = r2; it.row < r_rows; it.next()) {
        Turn x = turned(it);
        store_turned(x, it.row);
    }
    if (tid == 0) *scale_at = s;
}

}  // namespace gqla
