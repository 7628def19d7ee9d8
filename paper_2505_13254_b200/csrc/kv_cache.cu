// hs_kv_append, hs_kv_append_path, hs_kv_read: keys and values into the pages of an eight-bit cache and back.
//
// An item is the key and the value of one (row, kv head), eight lanes each, so that a warp has two items a step: a lane has 16 of the 128 values, 16 bytes from
// every stretch of 128 bytes.  Writing, the largest magnitude of the eight lanes comes from shuffles of the bits of |x| (they order like the values, infinities and NaN
// on top), the scale's exponent from its bits; reading is the way back.  Bound by HBM: an item reads 512 (bf16) or 1024 bytes and writes 258.  That takes few
// instructions a byte (with 16 lanes a row and eight values a lane the rows of eight prompts took 64 us in place of 29) and many loads in flight: 152 MB of
// appends 30 us, 5.1 TB/s; 499 MB of reads 81 us, 6.2 TB/s.
#include <cuda_bf16.h>

#include "hs_common.cuh"
#include "hs_layout.h"
#include "hs_ptx.cuh"
#include "kv_page.cuh"

#define KV_THREADS 256
// Steps a warp has in flight.  Appends of eight prompts (152 MB) and reads of long prefixes (499 MB) take 32 and 100 us with one, 29 and 81 with two, 31 and 82 with
// four, 39 and 83 with eight; small calls 5.7 us with one or two, 7 with eight.
#define KV_STEPS 2

struct AppendRows {                 // rows by offsets
    const int* row_off;
    int n_rows;
};
struct AppendPath {                 // rows of the accepted path
    const int* pruned_status;
    const int* accept_status;
    const int* accept_len;
    const int* path;                // path_compact or path_nodes
    const int* row_base;            // keep_off or node_off
    const int* n_keep;
    int path_cap, max_rows, compact;
};

// A lane's 16 values of a row: 16 bytes of each stretch of 128 (two of bf16, four of fp32).
template <typename T> struct KvRow;
template <> struct KvRow<__nv_bfloat16> {
    uint4 w[2];
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int sub) {
        w[0] = ld_stream(reinterpret_cast<const uint4*>(row) + sub);
        w[1] = ld_stream(reinterpret_cast<const uint4*>(row) + 8 + sub);
    }
    // bits of the largest magnitude
    __device__ __forceinline__ unsigned int amax() const {
        unsigned int a = 0u;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(a) : "r"((&w[c].x)[i] & 0x7fff7fffu));
        return max(a << 16, a & 0xffff0000u);
    }
    __device__ __forceinline__ void write(unsigned char* row, int sub, float f) const {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            auto pair = [&](unsigned int x) { return e4m3_pair(bf16_lo(x) * f, bf16_hi(x) * f); };
            *reinterpret_cast<uint2*>(row + c * 64 + sub * 8) = make_uint2(pair(w[c].x) | pair(w[c].y) << 16, pair(w[c].z) | pair(w[c].w) << 16);
        }
    }
};
template <> struct KvRow<float> {
    uint4 w[4];
    __device__ __forceinline__ void load(const float* row, int sub) {
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = ld_stream(reinterpret_cast<const uint4*>(row) + 8 * c + sub);
    }
    __device__ __forceinline__ unsigned int amax() const {
        unsigned int a = 0u;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) a = max(a, (&w[c].x)[i] & 0x7fffffffu);
        return a;
    }
    __device__ __forceinline__ void write(unsigned char* row, int sub, float f) const {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<unsigned int*>(row + c * 32 + sub * 4) = e4m3_pair(__uint_as_float(w[c].x) * f, __uint_as_float(w[c].y) * f) |
                                                                       e4m3_pair(__uint_as_float(w[c].z) * f, __uint_as_float(w[c].w) * f) << 16;
    }
};

// the row's eight lanes quantise it and store 128 bytes and the scale byte (row < 0: nowhere)
template <typename T>
__device__ __forceinline__ void write_row(const KvPages& c, long long row, bool is_v, int sub, const KvRow<T>& x) {
    unsigned int a = x.amax();
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(HS_FULL_MASK, a, o));
    if (row < 0) return;
    const unsigned int s = e8m0_of(a);
    unsigned char* to = (is_v ? c.v : c.k) + row * HS_HEAD_DIM;
    if (s != 255u) x.write(to, sub, e8m0_inverse(s));
    else *reinterpret_cast<uint4*>(to + sub * 16) = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
    if (sub == 0) (is_v ? c.v_scale : c.k_scale)[row] = (unsigned char)s;
}

// A lane's bytes of a row and its values.
template <typename T> struct KvBytes;
template <> struct KvBytes<__nv_bfloat16> {
    uint2 w[2];
    __device__ __forceinline__ void load(const unsigned char* row, int sub) {
        w[0] = *reinterpret_cast<const uint2*>(row + sub * 8);
        w[1] = *reinterpret_cast<const uint2*>(row + 64 + sub * 8);
    }
    __device__ __forceinline__ void write(__nv_bfloat16* row, int sub, float f) const {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            auto pair = [&](unsigned int x) {
                const float2 v = e4m3_floats(x);
                __nv_bfloat162 h = __floats2bfloat162_rn(v.x * f, v.y * f);      // exact: four significant bits (below 2^-130 rounded to a multiple of 2^-133)
                return *reinterpret_cast<unsigned int*>(&h);
            };
            *(reinterpret_cast<uint4*>(row) + c * 8 + sub) = make_uint4(pair(w[c].x), pair(w[c].x >> 16), pair(w[c].y), pair(w[c].y >> 16));
        }
    }
};
template <> struct KvBytes<float> {
    unsigned int w[4];
    __device__ __forceinline__ void load(const unsigned char* row, int sub) {
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = *reinterpret_cast<const unsigned int*>(row + c * 32 + sub * 4);
    }
    __device__ __forceinline__ void write(float* row, int sub, float f) const {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float2 a = e4m3_floats(w[c]), b = e4m3_floats(w[c] >> 16);
            *(reinterpret_cast<float4*>(row) + c * 8 + sub) = make_float4(a.x * f, a.y * f, b.x * f, b.y * f);
        }
    }
};

// The items of a half of a warp: first, first + 2, ..  Rows and heads of an item.
struct ItemWalk {
    unsigned int item, row, head;
    __device__ __forceinline__ ItemWalk(unsigned int first, int hkv) : item(first), row(first / (unsigned int)hkv), head(first - row * (unsigned int)hkv) {}
    // (true: another row)
    __device__ __forceinline__ bool next(int hkv) {
        item += 2;
        head += 2;
        if (head < (unsigned int)hkv) return false;
        head -= hkv;
        ++row;
        if (head >= (unsigned int)hkv) { head -= hkv; ++row; }      // (one head)
        return true;
    }
};

// Lengths behind the call, by a block of their own: `rows(b)` of them asked for.
template <typename Rows>
__device__ __forceinline__ bool write_lengths(const KvPages& c, int* len_out, Rows rows) {
    if (!len_out || blockIdx.x != gridDim.x - 1) return false;
    const int cap = c.max_pages << c.log_page;
    for (int b = threadIdx.x; b < c.batch; b += blockDim.x) {
        const int n = kv_length(c, b);
        len_out[b] = n + min(max(rows(b), 0), cap - n);
    }
    return true;
}

template <typename T>
__global__ void __launch_bounds__(KV_THREADS)
kv_append_kernel(const KvPages c, const AppendRows a, const T* __restrict__ k, const T* __restrict__ v, const long long token_stride,
                 const long long head_stride, int* len_out) {
    pdl_launch_dependents();
    pdl_wait();
    // (rows that the offsets name behind the arrays are none)
    if (blockIdx.x == 0 && threadIdx.x == 0 && (a.row_off[c.batch] > a.n_rows || a.row_off[0] < 0)) atomicCAS(c.err, 0, (int)HS_ERR_SHAPE);
    if (write_lengths(c, len_out, [&](int b) { return min(a.row_off[b + 1], a.n_rows) - min(a.row_off[b], a.n_rows); })) return;
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const bool is_v = lane & 8;
    const unsigned int first = (blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5)) * (2 * KV_STEPS), total = (unsigned int)a.n_rows * (unsigned int)c.hkv;
    if (first >= total) return;
    const ItemWalk start(first + (lane >> 4), c.hkv);
    const T* from = is_v ? v : k;
    KvRow<T> x[KV_STEPS];
    {
        ItemWalk w = start;
#pragma unroll
        for (int i = 0; i < KV_STEPS; ++i) {
            if (w.item < total) x[i].load(from + (long long)w.row * token_stride + (long long)w.head * head_stride, sub);
            w.next(c.hkv);
        }
    }
    ItemWalk w = start;
    int b = seq_of_row(a.row_off, c.batch, (int)(first / (unsigned int)c.hkv), lane);
    long long at = -1;
    bool fresh = true;                                             // `at` is not this row's yet
#pragma unroll
    for (int i = 0; i < KV_STEPS; ++i) {
        if (fresh && w.item < total) {
            const int row = (int)w.row;
            while (b < c.batch && row >= a.row_off[b + 1]) ++b;
            at = -1;
            if (b < c.batch && row >= a.row_off[b]) {              // (rows behind the last sequence go nowhere)
                const long long pos = (long long)kv_length(c, b) + (row - a.row_off[b]);
                if (pos < ((long long)c.max_pages << c.log_page)) at = kv_row(c, b, (int)pos);
                else kv_bad_page(c.err);
            }
        }
        write_row(c, at < 0 || w.item >= total ? -1 : at + ((long long)w.head << c.log_page), is_v, sub, x[i]);
        fresh = w.next(c.hkv);
    }
}

__global__ void __launch_bounds__(KV_THREADS)
kv_append_path_kernel(const KvPages c, const AppendPath a, const __nv_bfloat16* __restrict__ k, const __nv_bfloat16* __restrict__ v, int* len_out) {
    pdl_launch_dependents();
    pdl_wait();
    auto tokens = [&](int b) {                                     // (one round trip)
        const int failed = a.pruned_status[b] | a.accept_status[b], n = a.accept_len[b] + 1;
        if (failed != 0) return 0;
        if (n > a.path_cap) kv_bad_page(c.err);
        return min(max(n, 0), a.path_cap);
    };
    if (write_lengths(c, len_out, tokens)) return;
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const bool is_v = lane & 8;
    const unsigned int item = (blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5)) * 2u + (lane >> 4);
    const unsigned int slot = item / (unsigned int)c.hkv, b = slot / (unsigned int)a.path_cap;
    const int head = (int)(item - slot * (unsigned int)c.hkv), i = (int)(slot - b * (unsigned int)a.path_cap);
    KvRow<__nv_bfloat16> x;
    long long at = -1;
    if (b < (unsigned int)c.batch) {
        // one round trip for what says whether and where there is a row
        const int n = tokens(b), node = a.path[(size_t)b * a.path_cap + i], base = a.row_base[b], nodes = a.compact ? a.n_keep[b] : a.row_base[b + 1] - base;
        const long long row = (long long)base + node, pos = (long long)kv_length(c, b) + i;
        const bool there = node >= 0 && node < nodes && row >= 0 && row < a.max_rows;
        if (i < n && there) {
            x.load((is_v ? v : k) + (row * c.hkv + head) * HS_HEAD_DIM, sub);
            if (pos < ((long long)c.max_pages << c.log_page)) at = kv_row(c, b, (int)pos);
            else kv_bad_page(c.err);
        } else if (i < n) {
            kv_bad_page(c.err);                                    // not a path of this tree, or of these rows: its token stays unwritten
        }
    }
    if (at < 0) x.w[0] = x.w[1] = make_uint4(0u, 0u, 0u, 0u);
    write_row(c, at < 0 ? -1 : at + ((long long)head << c.log_page), is_v, sub, x);
}

template <typename T>
__global__ void __launch_bounds__(KV_THREADS)
kv_read_kernel(const KvPages c, const int* __restrict__ row_off, const int* __restrict__ start, const int n_rows, T* __restrict__ k,
               T* __restrict__ v, const long long token_stride, const long long head_stride) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const bool is_v = lane & 8;
    const unsigned int first = (blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5)) * (2 * KV_STEPS), total = (unsigned int)n_rows * (unsigned int)c.hkv;
    if (first >= total) return;
    const ItemWalk begin(first + (lane >> 4), c.hkv);
    int b = seq_of_row(row_off, c.batch, (int)(first / (unsigned int)c.hkv), lane);
    const unsigned char *from = is_v ? c.v : c.k, *scales = is_v ? c.v_scale : c.k_scale;
    KvBytes<T> x[KV_STEPS];
    unsigned int s[KV_STEPS];                                         // the scale byte; 256: nothing to write
    {
        ItemWalk w = begin;
        long long at = -1;
        bool fresh = true;
#pragma unroll
        for (int i = 0; i < KV_STEPS; ++i) {
            if (fresh && w.item < total) {
                const int row = (int)w.row;
                while (b < c.batch && row >= row_off[b + 1]) ++b;
                at = -1;
                if (b < c.batch && row >= row_off[b]) {
                    const long long pos = (long long)(start ? start[b] : 0) + (row - row_off[b]);
                    if (pos >= 0 && pos < kv_length(c, b)) at = kv_row(c, b, (int)pos);
                }
            }
            s[i] = 256u;
            if (at >= 0 && w.item < total) {
                const long long r = at + ((long long)w.head << c.log_page);
                x[i].load(from + r * HS_HEAD_DIM, sub);
                s[i] = scales[r];
            }
            fresh = w.next(c.hkv);
        }
    }
    ItemWalk w = begin;
    T* to = is_v ? v : k;
#pragma unroll
    for (int i = 0; i < KV_STEPS; ++i) {
        if (s[i] < 256u) x[i].write(to + (long long)w.row * token_stride + (long long)w.head * head_stride, sub, e8m0_value(s[i]));
        w.next(c.hkv);
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------
// blocks for items, and one for the lengths
static unsigned int blocks_of(long long items, int steps, bool lengths) {
    const long long per = (long long)(KV_THREADS / 32) * 2 * steps;
    return (unsigned int)((items + per - 1) / per) + (lengths ? 1u : 0u);
}

hs_status hs_launch_kv_append(hs_ctx* ctx, const hs_kv_cache* cache, const void* k, const void* v, hs_dtype dtype,
                              int64_t token_stride, int64_t head_stride, const int32_t* row_off, int32_t n_rows,
                              int32_t* len_out, cudaStream_t stream) {
    const KvPages c = kv_pages(cache, ctx->counters + HS_CNT_ERROR);
    const AppendRows a{row_off, n_rows};
    const long long items = (long long)n_rows * cache->hkv;
    if (items > 0x7fffffffll) return HS_ERR_SHAPE;
    // (without rows the offsets are looked at all the same)
    const dim3 grid(max(blocks_of(items, KV_STEPS, len_out != nullptr), 1u)), block(KV_THREADS), one(1, 1, 1);
    const long long ts = token_stride, hs = head_stride;
    cudaError_t e;
    if (dtype == HS_BF16)
        e = hs_launch(kv_append_kernel<__nv_bfloat16>, grid, block, 0, stream, ctx->pdl, one, c, a, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, ts, hs, len_out);
    else
        e = hs_launch(kv_append_kernel<float>, grid, block, 0, stream, ctx->pdl, one, c, a, (const float*)k, (const float*)v, ts, hs, len_out);
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}

hs_status hs_launch_kv_append_path(hs_ctx* ctx, const hs_kv_cache* cache, const hs_pruned_tree* pruned,
                                   const hs_accept_out* accept, int32_t layout, const int32_t* node_off, const void* k_tree,
                                   const void* v_tree, int32_t max_rows, int32_t* len_out, cudaStream_t stream) {
    const KvPages c = kv_pages(cache, ctx->counters + HS_CNT_ERROR);
    const bool compact = layout == HS_ROWS_COMPACT;
    AppendPath a;
    a.pruned_status = pruned->status;
    a.accept_status = accept->status;
    a.accept_len = accept->accept_len;
    a.path = compact ? accept->path_compact : accept->path_nodes;
    a.row_base = compact ? pruned->keep_off : node_off;
    a.n_keep = pruned->n_keep;
    a.path_cap = accept->path_cap;
    a.max_rows = max_rows;
    a.compact = compact;
    const long long items = (long long)cache->batch * accept->path_cap * cache->hkv;
    if (items > 0x7fffffffll) return HS_ERR_SHAPE;
    const cudaError_t e = hs_launch(kv_append_path_kernel, dim3(blocks_of(items, 1, len_out != nullptr)), dim3(KV_THREADS), 0, stream, ctx->pdl, dim3(1, 1, 1), c, a,
                                    (const __nv_bfloat16*)k_tree, (const __nv_bfloat16*)v_tree, len_out);
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}

hs_status hs_launch_kv_read(hs_ctx* ctx, const hs_kv_cache* cache, const int32_t* row_off, const int32_t* first,
                            int32_t n_rows, void* k_out, void* v_out, hs_dtype dtype, int64_t token_stride,
                            int64_t head_stride, cudaStream_t stream) {
    const KvPages c = kv_pages(cache, ctx->counters + HS_CNT_ERROR);
    const long long items = (long long)n_rows * cache->hkv;
    if (items > 0x7fffffffll) return HS_ERR_SHAPE;
    const dim3 grid(blocks_of(items, KV_STEPS, false)), block(KV_THREADS), one(1, 1, 1);
    const long long ts = token_stride, hs = head_stride;
    cudaError_t e;
    if (dtype == HS_BF16)
        e = hs_launch(kv_read_kernel<__nv_bfloat16>, grid, block, 0, stream, ctx->pdl, one, c,
                      row_off, first, n_rows, (__nv_bfloat16*)k_out, (__nv_bfloat16*)v_out, ts, hs);
    else
        e = hs_launch(kv_read_kernel<float>, grid, block, 0, stream, ctx->pdl, one, c, row_off, first,
                      n_rows, (float*)k_out, (float*)v_out, ts, hs);
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}
