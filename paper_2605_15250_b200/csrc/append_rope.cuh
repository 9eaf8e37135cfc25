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
    // Sequence that owns new row i, and the row's position in it (negative: in front of the sequence, the row is skipped).
    __device__ __forceinline__ int32_t seq_of(int32_t i) const {
        int32_t lo = 0, hi = B - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (start[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
    __device__ __forceinline__ int32_t first_pos(int32_t b) const { return seqlens[b] - (start[b + 1] - start[b]); }
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

// A rotation item.  VEC: sixteen elements, item i of d_r / 16: the chunks 2 i and 2 i + 1, or i and i + d_r / 16 with halves.
// Otherwise: one pair, item i of d_r / 2.
template <bool VEC>
struct RopeItem {
    static constexpr int kN = VEC ? 8 : 1;  // elements of each of the two parts
    static __host__ __device__ int count(int d_r) { return VEC ? d_r / 16 : d_r / 2; }
    float a[kN], b[kN];
    int ca, cb;  // first columns of the parts
    __device__ __forceinline__ RopeItem(const RopeTable& t, int i)
        : ca(t.halves ? i * kN : 2 * i * kN), cb(t.halves ? i * kN + t.d_r / 2 : (2 * i + 1) * kN) {}
    template <typename T>
    __device__ __forceinline__ void load(const T* x) {
        if constexpr (VEC) {
            load8(x + ca, a);
            load8(x + cb, b);
        } else {
            a[0] = ldf(x + ca);
            b[0] = ldf(x + cb);
        }
    }
    __device__ __forceinline__ void rotate(const RopeTable& t, int32_t pos) {
        const float* cs = t.cs + (int64_t)pos * t.d_r;
        const int half = t.d_r / 2;
        if constexpr (VEC) {
            float c[8], s[8];
            if (t.halves) {
                load8(cs + ca, c);
                load8(cs + half + ca, s);
#pragma unroll
                for (int k = 0; k < 8; ++k) turn(a[k], b[k], c[k], s[k]);
            } else {  // pairs within each part: frequencies ca / 2 .. ca / 2 + 7 over both
                load8(cs + ca / 2, c);
                load8(cs + half + ca / 2, s);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    turn(a[2 * k], a[2 * k + 1], c[k], s[k]);
                    turn(b[2 * k], b[2 * k + 1], c[4 + k], s[4 + k]);
                }
            }
        } else {
            const int f = t.halves ? ca : ca / 2;
            turn(a[0], b[0], cs[f], cs[half + f]);
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* y) const {
        if constexpr (VEC) {
            store8(y + ca, a);
            store8(y + cb, b);
        } else {
            stf(y + ca, a[0]);
            stf(y + cb, b[0]);
        }
    }
};

// The queries' share of a launch: item index `i` counts (row, head, rotation item).
template <typename T, bool VEC>
__device__ __forceinline__ void rotate_queries(const NewRows& nr, const RopeTable& rope, const QueryRows& q, int64_t i, int32_t* status) {
    const int per = RopeItem<VEC>::count(rope.d_r);
    if (i >= nr.n * q.h_q * per) return;
    const int item = (int)(i % per), head = (int)(i / per % q.h_q);
    const int32_t tok = (int32_t)(i / per / q.h_q);
    const int32_t b = nr.seq_of(tok), pos = nr.first_pos(b) + tok - nr.start[b];
    if (pos < 0) return;
    if (pos >= rope.rows) return append_error(status, 1);
    RopeItem<VEC> x(rope, item);
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
    int32_t* status;
};

constexpr int kAppendMostRows = 8;  // new rows of a warp

// Item i, i + step, i + 2 step, .. of rows of `per` items each, without a division per item.
struct RowItems {
    int row, col, row_step, col_step, per;
    __device__ __forceinline__ RowItems(int i, int step, int per_)
        : row(i / per_), col(i % per_), row_step(step / per_), col_step(step % per_), per(per_) {}
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
// at a time (49000 rows of 1152 bytes: 41.7 us with a block per sixteen rows and one vector a thread in flight), the RoPE parts rotated an
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
    RowItems it(lane, 32, VEC ? a.r_kv * (int)sizeof(T) / 16 : a.r_kv);
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
        my_pos = a.nr.first_pos(b) + tok - a.nr.start[b];
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
    const int turns = RopeItem<VEC>::count(a.rope.d_r);
    for (int i0 = 0; i0 < n * turns; i0 += 32) {
        const int i = i0 + lane, k = turns > 0 ? i / turns : 0;
        const int64_t row = row_of(k);
        const int32_t pos = __shfl_sync(0xffffffffu, my_pos, k < n ? k : 0);
        if (k >= n || row < 0) continue;
        RopeItem<VEC> x(a.rope, i % turns);
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
// Largest finite magnitude of eight bf16 values, as the 15 bits that order like it, kept in both halves of `m`.  (Infinities and NaN
// are 0x7f80 and beyond; they are looked for only where the plain maximum says that there are some.)
__device__ __forceinline__ uint32_t bf16_max(uint32_t m, const uint4& u) {
    const uint32_t w[4] = {u.x & 0x7fff7fffu, u.y & 0x7fff7fffu, u.z & 0x7fff7fffu, u.w & 0x7fff7fffu};
    uint32_t x = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
    if (__vcmpgeu2(x, 0x7f807f80u) != 0) {
        x = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) x = __vmaxu2(x, w[i] & __vcmpltu2(w[i], 0x7f807f80u));
    }
    return __vmaxu2(m, x);
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
    int32_t* status;
};

// A block takes one head of one page that gets new rows.  Units of pages, without a prefix sum over the sequences:
//   by rows    unit u is new row u, if that is the first new one of its page (steps: fewer rows than the other bound)
//   otherwise  unit u of sequence b is its page number u - unit0(b) from the first touched one on, unit0(b) = (start[b] >> k) + 2 b
//              with 2^k <= page: n new rows touch at most (n - 1) / page + 2 pages, and successive unit0 are at least that far apart.
// What is left over exits.
// The first eight chunks of a thread stay in registers between the maximum and the coding: all of a page of 64 latent rows
// with 512 threads, of 64 rows of one head of a plane with 128; larger pages read the rest again, from L1 or L2.  (256 threads with
// sixteen chunks each left one block per SM: 20000 rows into the planes 205 us, a step of 64 rows 43.)
constexpr int kLatentThreads = 512, kPlaneThreads = 128;
template <typename T, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) append_fp8_kernel(const AppendFp8Args a) {
    constexpr int kWarps = THREADS / 32;
    __shared__ float red[kWarps];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if ((int64_t)blockIdx.x >= a.kv_blocks)
        return rotate_queries<T, VEC>(a.nr, a.rope, a.q, ((int64_t)blockIdx.x - a.kv_blocks) * THREADS + threadIdx.x, a.status);
    const int32_t unit = (int32_t)(blockIdx.x / a.heads_in_all);
    int head = (int)(blockIdx.x % a.heads_in_all);
    const int page = a.page_size;
    const int32_t b = a.unit_shift < 0 ? warp_last(a.nr.B, unit, [&](int32_t i) { return a.nr.start[i]; })
                                       : warp_last(a.nr.B, unit, [&](int32_t i) { return (a.nr.start[i] >> a.unit_shift) + 2 * i; });
    const int32_t s0 = a.nr.start[b], n = a.nr.start[b + 1] - s0;
    const int32_t T_len = a.nr.seqlens[b], first = T_len - n;
    if (n <= 0 || T_len <= 0) return;
    int32_t k;  // page of the sequence
    if (a.unit_shift < 0) {
        const int32_t pos = first + unit - s0;
        if (pos < 0 || (unit != s0 && pos % page != 0)) return;
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
    while (head >= a.plane[pl].heads) head -= a.plane[pl++].heads;
    const Fp8Plane& P = a.plane[pl];
    const T* src = (const T*)P.a + (int64_t)(s0 + lo - first) * P.a_stride + head * P.a_width;
    const T* rsrc = (const T*)a.k_r + (int64_t)(s0 + lo - first) * a.k_r_stride;
    const int width = P.a_width + (P.rope_heads ? a.rope.d_r : 0);
    const int rows = hi - lo;
    const int chunks = VEC ? P.a_width / 8 : P.a_width, turns = P.rope_heads ? RopeItem<VEC>::count(a.rope.d_r) : 0;
    const int tid = threadIdx.x;

    // largest finite magnitude of the new rows
    constexpr int kHeld = VEC && sizeof(T) == 2 ? 8 : 0;
    constexpr int kElems = VEC ? 8 : 1;
    uint4 held[kHeld > 0 ? kHeld : 1];
    float amax = 0.f;
    const RowItems a0(tid, THREADS, chunks > 0 ? chunks : 1);
    const int a_rows = chunks > 0 ? rows : 0;
    if constexpr (kHeld > 0) {
        RowItems it = a0;
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            if (it.row < a_rows) held[h] = *reinterpret_cast<const uint4*>(src + (int64_t)it.row * P.a_stride + it.col * 8);
            it.next();
        }
    }
    const RowItems r0(tid, THREADS, turns > 0 ? turns : 1);
    const int r_rows = turns > 0 ? rows : 0;
    if (pid < 0 || pid >= a.n_pages) {
        if (tid == 0) append_error(a.status, 2);
        return;
    }
    e4m3* page_dst = (e4m3*)P.dst + (int64_t)pid * page * P.dst_stride + (int64_t)head * width;
    e4m3* dst = page_dst + (int64_t)(lo - p0) * P.dst_stride;
    float* const scale_at = P.scale + (int64_t)pid * P.heads + head;
    const float s_old = lo > p0 ? *scale_at : 0.f;  // the page's older rows, if it has any, hold it to this
    {
        RowItems it = a0;
        if constexpr (kHeld > 0) {
            uint32_t top = 0;
#pragma unroll
            for (int h = 0; h < kHeld; ++h) {
                if (it.row < a_rows) top = bf16_max(top, held[h]);
                it.next();
            }
            amax = fmaxf(amax, __uint_as_float(__vmaxu2(top, top >> 16) << 16));
        }
        for (; it.row < a_rows; it.next()) {
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
        for (it = r0; it.row < r_rows; it.next()) {
            RopeItem<VEC> x(a.rope, it.col);
            x.load(rsrc + (int64_t)it.row * a.k_r_stride);
            x.rotate(a.rope, lo + it.row);
#pragma unroll
            for (int e = 0; e < RopeItem<VEC>::kN; ++e) amax = finite_max(finite_max(amax, x.a[e]), x.b[e]);
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
        for (RowItems it(tid, THREADS, VEC ? width / 8 : width); it.row < lo - p0; it.next()) {
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
    RowItems it = a0;
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            if (it.row < a_rows) {
                float v[8];
                unpack8(held[h], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= inv;
                store8(dst + (int64_t)it.row * P.dst_stride + it.col * 8, v);
            }
            it.next();
        }
    }
    for (; it.row < a_rows; it.next()) {
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
    for (it = r0; it.row < r_rows; it.next()) {
        RopeItem<VEC> x(a.rope, it.col);
        x.load(rsrc + (int64_t)it.row * a.k_r_stride);
        x.rotate(a.rope, lo + it.row);
#pragma unroll
        for (int e = 0; e < RopeItem<VEC>::kN; ++e) {
            x.a[e] *= inv;
            x.b[e] *= inv;
        }
        x.store(dst + (int64_t)it.row * P.dst_stride + P.a_width);
    }
    if (tid == 0) *scale_at = s;
}

}  // namespace gqla
