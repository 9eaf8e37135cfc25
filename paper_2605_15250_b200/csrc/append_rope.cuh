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
    int32_t per_block, kv_blocks;  // new rows of a block; blocks behind kv_blocks rotate queries
    int32_t* status;
};

constexpr int kAppendMostRows = 16;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kAppendThreads) append_rope_kernel(const AppendArgs a) {
    __shared__ int64_t dst_row[kAppendMostRows];
    __shared__ int32_t position[kAppendMostRows];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if ((int)blockIdx.x >= a.kv_blocks)
        return rotate_queries<T, VEC>(a.nr, a.rope, a.q, (int64_t)(blockIdx.x - a.kv_blocks) * kAppendThreads + threadIdx.x, a.status);
    const int64_t tok0 = (int64_t)blockIdx.x * a.per_block;
    const int n = (int)(a.nr.n - tok0 < a.per_block ? a.nr.n - tok0 : a.per_block);
    if ((int)threadIdx.x < n) {
        const int32_t tok = (int32_t)tok0 + threadIdx.x, b = a.nr.seq_of(tok);
        const int32_t pos = a.nr.first_pos(b) + tok - a.nr.start[b];
        int64_t row = -1;
        if (pos >= a.rope.rows && a.rope.d_r > 0) append_error(a.status, 1);
        else if (pos >= 0) row = checked_row(a.rows, b, pos, a.cache_rows, a.status);
        dst_row[threadIdx.x] = row;
        position[threadIdx.x] = pos;
    }
    __syncthreads();
    const int copies = VEC ? a.r_kv / 8 : a.r_kv;
    const int items = copies + RopeItem<VEC>::count(a.rope.d_r);
    for (int i = threadIdx.x; i < n * items; i += kAppendThreads) {
        const int k = i / items, it = i % items;
        if (dst_row[k] < 0) continue;
        const T* c = (const T*)a.c + (tok0 + k) * a.c_stride;
        T* y = (T*)a.cache + dst_row[k] * a.cache_stride;
        if (it < copies) {
            if constexpr (VEC) {
                constexpr int kVecs = sizeof(T) / 2;  // 16-byte vectors of eight elements
#pragma unroll
                for (int v = 0; v < kVecs; ++v)
                    reinterpret_cast<uint4*>(y + it * 8)[v] = reinterpret_cast<const uint4*>(c + it * 8)[v];
            } else {
                y[it] = c[it];
            }
        } else {
            RopeItem<VEC> x(a.rope, it - copies);
            x.load((const T*)a.k_r + (tok0 + k) * a.k_r_stride);
            x.rotate(a.rope, position[k]);
            x.store(y + a.r_kv);
        }
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
    int32_t* status;
};

// A block takes one head of one page that gets new rows.  Unit u of sequence b is its page number u - unit0(b) from the first
// touched one on, unit0(b) = start[b] / page + 2 b: a sequence with n new rows touches at most (n - 1) / page + 2 pages, and
// successive unit0 are at least that far apart, so that no prefix sum over the sequences is needed; what is left over exits.
// The rows' first kHeld chunks per thread stay in registers between the maximum and the coding (64 rows of the latent
// cache are sixteen chunks a thread); larger pages read the rest again, from L1 or L2.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kAppendThreads) append_fp8_kernel(const AppendFp8Args a) {
    constexpr int kWarps = kAppendThreads / 32;
    __shared__ float red[kWarps];
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if ((int64_t)blockIdx.x >= a.kv_blocks)
        return rotate_queries<T, VEC>(a.nr, a.rope, a.q, ((int64_t)blockIdx.x - a.kv_blocks) * kAppendThreads + threadIdx.x, a.status);
    const int32_t unit = (int32_t)(blockIdx.x / a.heads_in_all);
    int head = (int)(blockIdx.x % a.heads_in_all);
    const int page = a.page_size;
    int32_t b = 0;
    {
        int32_t hi = a.nr.B - 1;
        while (b < hi) {
            const int32_t mid = (b + hi + 1) >> 1;
            if (a.nr.start[mid] / page + 2 * mid <= unit) b = mid;
            else hi = mid - 1;
        }
    }
    const int32_t s0 = a.nr.start[b], n = a.nr.start[b + 1] - s0;
    const int32_t T_len = a.nr.seqlens[b], first = T_len - n;
    if (n <= 0 || T_len <= 0) return;
    const int32_t k = (first > 0 ? first / page : 0) + unit - (s0 / page + 2 * b);  // page of the sequence
    if (k < 0 || (int64_t)k * page >= T_len) return;
    const int32_t p0 = k * page;
    const int32_t lo = p0 > first ? p0 : first;  // new rows [lo, hi) of this page; first < p0 + page by the choice of k
    int32_t hi = T_len - p0 < page ? T_len : p0 + page;
    const int32_t pid = k < a.max_pages ? a.block_table[(int64_t)b * a.max_pages + k] : -1;
    if (pid < 0 || pid >= a.n_pages) {
        if (threadIdx.x == 0) append_error(a.status, 2);
        return;
    }
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
    e4m3* page_dst = (e4m3*)P.dst + (int64_t)pid * page * P.dst_stride + (int64_t)head * width;
    e4m3* dst = page_dst + (int64_t)(lo - p0) * P.dst_stride;
    const int rows = hi - lo;
    const int chunks = VEC ? P.a_width / 8 : P.a_width, turns = P.rope_heads ? RopeItem<VEC>::count(a.rope.d_r) : 0;
    float* const scale_at = P.scale + (int64_t)pid * P.heads + head;
    const float s_old = lo > p0 ? *scale_at : 0.f;  // the page's older rows, if it has any, hold it to this
    const int tid = threadIdx.x;

    // largest finite magnitude of the new rows
    constexpr int kHeld = VEC && sizeof(T) == 2 ? 16 : 0;
    uint4 held[kHeld > 0 ? kHeld : 1];
    float amax = 0.f;
    const int a_items = rows * chunks;
    if constexpr (kHeld > 0) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = tid + h * kAppendThreads;
            if (i < a_items) held[h] = *reinterpret_cast<const uint4*>(src + (int64_t)(i / chunks) * P.a_stride + i % chunks * 8);
        }
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (tid + h * kAppendThreads < a_items) {
                float v[8];
                unpack8(held[h], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = finite_max(amax, v[e]);
            }
    }
    for (int i = tid + kHeld * kAppendThreads; i < a_items; i += kAppendThreads) {
        const T* x = src + (int64_t)(i / chunks) * P.a_stride + i % chunks * (VEC ? 8 : 1);
        if constexpr (VEC) {
            float v[8];
            load8(x, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = finite_max(amax, v[e]);
        } else {
            amax = finite_max(amax, ldf(x));
        }
    }
    for (int i = tid; i < rows * turns; i += kAppendThreads) {
        RopeItem<VEC> x(a.rope, i % turns);
        x.load(rsrc + (int64_t)(i / turns) * a.k_r_stride);
        x.rotate(a.rope, lo + i / turns);
#pragma unroll
        for (int e = 0; e < RopeItem<VEC>::kN; ++e) amax = finite_max(finite_max(amax, x.a[e]), x.b[e]);
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
        const int per = VEC ? width / 8 : width;
        for (int i = tid; i < (lo - p0) * per; i += kAppendThreads) {
            e4m3* y = page_dst + (int64_t)(i / per) * P.dst_stride + i % per * (VEC ? 8 : 1);
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
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int i = tid + h * kAppendThreads;
            if (i < a_items) {
                float v[8];
                unpack8(held[h], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= inv;
                store8(dst + (int64_t)(i / chunks) * P.dst_stride + i % chunks * 8, v);
            }
        }
    }
    for (int i = tid + kHeld * kAppendThreads; i < a_items; i += kAppendThreads) {
        const int r = i / chunks, c = i % chunks * (VEC ? 8 : 1);
        const T* x = src + (int64_t)r * P.a_stride + c;
        e4m3* y = dst + (int64_t)r * P.dst_stride + c;
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
    for (int i = tid; i < rows * turns; i += kAppendThreads) {
        RopeItem<VEC> x(a.rope, i % turns);
        x.load(rsrc + (int64_t)(i / turns) * a.k_r_stride);
        x.rotate(a.rope, lo + i / turns);
#pragma unroll
        for (int e = 0; e < RopeItem<VEC>::kN; ++e) {
            x.a[e] *= inv;
            x.b[e] *= inv;
        }
        x.store(dst + (int64_t)(i / turns) * P.dst_stride + P.a_width);
    }
    if (tid == 0) *scale_at = s;
}

}  // namespace gqla
