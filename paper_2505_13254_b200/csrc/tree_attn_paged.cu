// hs_tree_verify_attention_paged: tree-mask attention over a paged cache at eight bits, one launch.
//
//   out = softmax(scale q [K; K_tree]^T + mask) [V; V_tree],   K_t = byte * 2^(s_t - 127) in E4M3, the same for V
//
// CTA = (block of 32 to 256 query rows, KV split, sequence x kv head).  Query row r = node * G + g: the heads of a group and the kept nodes form the
// dense dimension.  The tiles of 64 keys - first the tree's one or two, then the prefix's - are shared out evenly over the splits, which form a cluster
// and merge through distributed shared memory.
//
// S = Q K^T takes the cached keys as they are (tcgen05.mma of kind::f8f6f4): a bf16 query is the sum of two E4M3 terms, q 2^-e = t1 + t2, its first four significant bits
// and its last four, so S is two products accumulated in fp32 and costs what bf16 would, without a conversion of K.  e puts a row's largest value into (224, 448]; what lies
// 2^9 below it or more is rounded to 2^-9, by at most 2^-17 of that value.  The keys' scales, powers of two, multiply the columns of S.  The tree's bf16 keys become
// two terms in the same way, and their S four products.
// O = P V has no such form: probabilities span more than eight bits can hold (a thousand keys of weight 2^-18 beside one of weight 1 matter).  So V's bytes become f16
// tiles in shared memory, exactly, and P is rounded to f16, eleven bits, all that is rounded on the way.  The values' scales go into the exponential's argument:
// P = 2^(t + B - R) with t the score in base 2, 2^B the token's scale and R the running maximum of t + B, so that O += P V' holds 2^-R sum 2^t V whatever the scales are, and the
// sum takes P 2^-B.  R follows what a row weighs, not what it masks or weighs with nothing: f16 keeps products of a weight and a token's values down to 2^-30 of the row's largest.
// Where the scales of a tile's tokens lie within 2^6 of one another, all of them take the largest (V' then carries the difference, exactly), B is one number a tile and goes into the
// exponential's multiply-add for nothing; that costs the bound 2^6.  Other tiles (rare in earnest: a token of next to no value among others) take a term, and an exponential for the sum, a score more:
// where every tile is one, four long trees take 620 us back to back in place of 362, 32 ragged tokens 89 in place of 80, a tree of 60 behind 2048 19.2 in place of 17.0.
//   - two warps ask for keys (TMA, a page at a time, 128-byte swizzle: operand tiles)
//   - eight warps in four groups ask for the values and the scale bytes of every fourth tile (bulk copies) and turn the values into a swizzled f16 tile: four bytes by two PRMT, shifts and masks, one product a pair with the row's
//     power of two; and the keys' scale bytes into floats
//   - two warps issue S = Q K^T and O += P V
//   - two warpgroups run two online softmax streams, thread = query row: S from tensor memory, maximum, exponentials in base 2, P back as the A
//     operand.  With 128 rows they take alternate tiles; with 256 each has a block of 128 rows and takes every tile (WIDE), so that a tile is
//     fetched and converted once for twice the rows.  Up to 64 or 32 rows stand in the 128 lanes two or four times (REP), and every copy takes its own half or
//     quarter of a tile's columns, with a maximum, a sum and an O of its own: a tile's softmax is as many times shorter, and all four schedulers
//     have a share of it.
// Registers: 640 threads are launched with 96 each; the softmax warps take 144, what the others give back.
// What bounds it.  Tokens without drafts: HBM, a tile of keys and values a CTA every 750 clocks of which 665 are the bytes' (32 sequences of 1024 to 8192 tokens, 307 MB: 80 us back to back,
// 3.8 TB/s with both CTAs' starts and ends; a CTA spends 12000 clocks on those).  Trees behind long prefixes: the softmax warps' instructions (four trees of 62 nodes and 64 heads behind
// 32768 tokens, 267 GFLOP: 362 us back to back, 0.74 PFLOP/s; an SM issues in 60% of its clocks, the exponential unit is busy in 42%, the products take 512 of a tile's 1300 clocks).  Small calls: the
// chain from the launch to the merged rows (one token behind 512: 7.7 us; a tree of 60 behind 2048: 16.5 us).
// Behind the last token and in the last page a tile is zero, whatever the memory holds, and masked.  A tree value that is not finite, or of 2^10 and more, is
// zero in the product (0 * inf would reach the rows that mask it, and a large one would cost the other columns of the rows that see it their bits) and added to the rows that see it at the end.
#include <cuda_fp16.h>
#include <math_constants.h>

#include <type_traits>

#include "hs_common.cuh"
#include "hs_layout.h"
#include "hs_ptx.cuh"
#include "kv_page.cuh"
#include "paged_choice.h"

#define PG_BM 128                                   // query rows of a stream's block
#define PG_BN 64
#define PG_TILE_BYTES (PG_BN * HS_HEAD_DIM * 2)     // 16 KiB: one f16 tile of V
#define PG_UNIT_BYTES (PG_BN * HS_HEAD_DIM)         // 8 KiB: K or V of a tile at eight bits
#define PG_KEYS 6                                   // tiles of K (a tree tile is two: its terms)
#define PG_GROUPS 4                                 // groups of converters, and f16 tiles of V
#define PG_EXPS 8                                   // tiles whose scales are kept
#define PG_FLAT 6                                   // a tile whose tokens' exponents differ by no more has one for all of them
#define PG_LIFT 6.f                                 // P = 2^(6 + ..): f16 then keeps weights down to 2^-30 of the largest
#define PG_ROW_STRIDE (HS_HEAD_DIM * 2 + 16)        // a pushed partial row: 128 f16 of O 2^-k, {max, sum, k}
#define PG_THREADS 640
#define PG_REGS 96                                  // of a thread at launch
#define PG_SM_THREADS 256                           // softmax threads: row = tid & 127, stream = tid >> 7
#define PG_CV_THREADS 64                            // converting threads of a group
#define PG_WARP_PV 16
#define PG_WARP_S 17
#define PG_WARP_LOAD 18                             // and 19
#define PG_TMEM_COLS 512                            // S of stream g: 64 g ..; O: 128 + 128 g ..; P: 384 + 32 g ..; Q: 448 ..
#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// Shared memory, from a 1024-byte boundary.  Up to 128 rows: the query block's place takes the partials that the cluster sends, once it is in tensor memory; 256 rows:
// the first block is staged there too, the second stays as an operand, and the partials go over the tiles, behind a barrier of the cluster.
template <int ROWS>
struct Layout {
    static constexpr bool WIDE = ROWS == 256;
    static constexpr int rows = WIDE ? 256 : 128;
    // units of V in flight (with four, 32 ragged sequences without drafts take 83 us instead of 80: their bytes take 2300 clocks to come)
    static constexpr int units = WIDE ? 4 : 8;
    static_assert(units % PG_GROUPS == 0 && PG_KEYS % 2 == 0, "a unit serves one group: two could not tell its barriers' rounds apart by their parity");
    static constexpr int recv_bytes = PG_ROW_STRIDE * (rows + 2 * PG_MAX_SPLIT);
    static constexpr int q_bytes = rows * HS_HEAD_DIM * 2;
    static constexpr int k = 0, unit = k + PG_KEYS * PG_UNIT_BYTES, v = unit + units * PG_UNIT_BYTES, q = v + PG_GROUPS * PG_TILE_BYTES;
    static constexpr int recv = WIDE ? k : q;
    static constexpr int scale = q + (!WIDE && recv_bytes > q_bytes ? recv_bytes : q_bytes);      // scale bytes of the units: V's 64, K's 64
    static constexpr int bar = scale + units * 2 * PG_BN;
    static constexpr int x = bar + 512;              // the streams' maxima and sums, [2][128] each
    static constexpr int exps = x + 4 * PG_BM * 4;   // per tile {B, 2^-B}, {0, 0} where the tokens have exponents of their own
    static constexpr int ks = exps + 2 * PG_EXPS * 4;     // per tile the keys' scales
    static constexpr int vs = ks + PG_EXPS * PG_BN * 4;   // and the tokens' exponents
    static constexpr int qs = vs + PG_EXPS * PG_BN * 2;   // the query rows' scales
    static constexpr int red = qs + rows * 4;             // largest and smallest exponents of the converting warps
    static constexpr int end = red + 64;
    static constexpr int part = k;                   // fewer rows than 128: the streams' partials, 128 rows of part_stride floats
    static constexpr int part_stride = HS_HEAD_DIM + 4;
    static_assert(PG_BM * part_stride * 4 <= q, "they lie over the tiles");
    static constexpr int bytes = end + 1024;
    static_assert(bytes <= 227 * 1024, "shared memory of one CTA");
    static_assert(!WIDE || recv + recv_bytes <= q, "the partials fit over the tiles");
    static_assert(scale % 16 == 0 && bar % 8 == 0 && exps % 8 == 0 && ks % 16 == 0 && recv % 16 == 0, "alignment");
};

struct PagedParams {
    KvPages c;
    const __nv_bfloat16 *q, *k_tree, *v_tree;
    __nv_bfloat16* out;
    float* lse_out;
    const int *n_keep, *keep_off, *keep_idx, *status, *node_off;
    const unsigned long long* anc_mask;
    int hq, G, layout, nsplit, max_nodes, max_rows;
    unsigned int inv_g;            // ceil(2^16 / G): r / G = r * inv_g >> 16 for the row numbers r < 2^11
    float scale_log2;
};

__device__ __forceinline__ unsigned int pg_pack(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<unsigned int*>(&v);
}
__device__ __forceinline__ unsigned int pg_pack_half(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<unsigned int*>(&v);
}
__device__ __forceinline__ float2 pg_halves(unsigned int w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
// byte offset of (row, 16-byte chunk 0..15 of the 128 d's) in a tile of `rows` rows with the 128-byte swizzle: two halves of 64 d's
__device__ __forceinline__ unsigned int pg_off(int rows, int row, int chunk) {
    return (unsigned int)((chunk >> 3) * (rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
}
// Four E4M3 bytes as f16 times 2^-8, exact, times a power of two: a byte's sign at bit 15, its exponent and mantissa at bits 13 .. 7 (f16's bias is 8 more), zeros and
// subnormals alike.  (cvt.rn.f16x2.e4m3x2 takes a scheduler 16 clocks: a unit took a group of four warps 1000 clocks with it.)
__device__ __forceinline__ uint2 e4m3_half4(unsigned int w, unsigned int two) {
    unsigned int a, b, c, d;                                 // a byte and its sign, eight times (__byte_perm takes no sign bytes)
    asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(a) : "r"(w));
    asm("prmt.b32 %0, %1, 0, 0xb3a2;" : "=r"(b) : "r"(w));
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(c) : "r"(a * 128u & 0xbf80bf80u), "r"(two));
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(b * 128u & 0xbf80bf80u), "r"(two));
    return make_uint2(c, d);
}
// A pair of bf16 of at most 448 in magnitude as two E4M3 terms: the value times 2^-120 has the byte's exponent and mantissa at bits 10 .. 4 (bf16's bias is 120 more), the
// first four significant bits are the first term, what is left, exactly, has four more; where those pass E4M3's last bit, 2^-9, they are rounded to it.
__device__ __forceinline__ void e4m3_terms(unsigned int w, unsigned int two, unsigned int& t1, unsigned int& t2) {
    unsigned int y, r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(w), "r"(two));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(y), "r"(0x03800380u));      // 2^-120
    t1 = y & 0x87f087f0u;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(y), "r"(t1));
    t2 = (r + 0x00080008u) & 0x87f087f0u;
}
// the bytes of two pairs
__device__ __forceinline__ unsigned int e4m3_bytes(unsigned int a, unsigned int b) {
    a = (a >> 4 & 0x007f007fu) | (a >> 8 & 0x00800080u);
    b = (b >> 4 & 0x007f007fu) | (b >> 8 & 0x00800080u);
    return __byte_perm(a, b, 0x6420);
}
// 2^d twice in f16, d <= 15
__device__ __forceinline__ unsigned int half2_power(int d) {
    const unsigned int bits = d >= -14 ? (unsigned int)(15 + d) << 10 : d >= -24 ? 1u << (d + 24) : 0u;
    return bits * 0x10001u;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 16 bytes from global into shared memory, asynchronously; zeros where there is no source
__device__ __forceinline__ void copy16(unsigned int dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}
// The exponent of a token whose scale byte (or that of its largest |x|) is s: at least -60, so that sums of P 2^-B stay far inside fp32.
#define PG_SMALLEST 67u
__device__ __forceinline__ int token_exponent(unsigned int s) { return (int)max(s, PG_SMALLEST) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }
// bits of the larger |.| of a pair of bf16, as fp32
__device__ __forceinline__ unsigned int pair_amax(unsigned int w) { return max(w << 16 & 0x7fff0000u, w & 0x7fff0000u); }
__device__ __forceinline__ unsigned int pair_max(unsigned int a, unsigned int b) {
    asm("max.u16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
}
__device__ __forceinline__ unsigned int pair_min(unsigned int a, unsigned int b) {
    asm("min.u16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
}
// A tree value of 2^10 or more, an infinity or a NaN stays out of the product: what it would cost the other columns, or put into rows that mask it, it is added
// to the rows that see it at the end.  Its token counts as 2^10, so that R is at least t - 6 there and the weight 2^(t + 6 - R) at most 2^12, whatever is left of the token.  A pair without such values:
#define PG_APART 0x44800000u                        // 2^10, the bits
#define PG_ENDLESS 0x71800000u                      // 2^100: up to it the sum of 128 keys of such weights stays in fp32; from it on a value counts as infinite
__device__ __forceinline__ unsigned int near_or_zero(unsigned int w) {
    return ((w << 16 & 0x7fff0000u) >= PG_APART ? 0u : w & 0xffffu) | ((w & 0x7fff0000u) >= PG_APART ? 0u : w & 0xffff0000u);
}
// a pair of bf16 times f, as f16
__device__ __forceinline__ unsigned int scaled_half2(unsigned int w, float f) { return pg_pack_half(bf16_lo(w) * f, bf16_hi(w) * f); }
__device__ __forceinline__ void tmem_st8(unsigned int taddr, const unsigned int* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ float2 mul2_ftz(float2 a, float2 b) {
    unsigned long long ra, rb, rd;
    float2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(ra) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(rb) : "f"(b.x), "f"(b.y));
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(rd) : "l"(ra), "l"(rb));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(rd));
    return d;
}
__device__ __forceinline__ void tma_load_2d(unsigned int dst, const CUtensorMap* tm, int c0, int c1, unsigned int bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
// Instruction descriptor of kind::f8f6f4 with E4M3 operands, fp32 accumulation; D[tmem] (+)= A B with K = 32: A from tensor memory (four bytes a column, eight columns) or from
// shared memory.
__device__ __forceinline__ unsigned int umma_idesc_e4m3(int m, int n) {
    return (1u << 4) | ((unsigned int)(n >> 3) << 17) | ((unsigned int)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_ts_e4m3(unsigned int d_tmem, unsigned int a_tmem, unsigned long long b_desc, unsigned int idesc, unsigned int accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n\t}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u), "r"(0u), "r"(0u), "r"(0u)
        : "memory");
}
__device__ __forceinline__ void umma_ss_e4m3(unsigned int d_tmem, unsigned long long a_desc, unsigned long long b_desc, unsigned int idesc, unsigned int accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, {%5, %6, %7, %8}, p;\n\t}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u), "r"(0u), "r"(0u), "r"(0u)
        : "memory");
}
// D[tmem] (+)= A B of kind::f16 with f16 operands, fp32 accumulation
__device__ __forceinline__ unsigned int umma_idesc_half(int m, int n, bool b_mn_major) {
    return (1u << 4) | (b_mn_major ? (1u << 16) : 0u) | ((unsigned int)(n >> 3) << 17) | ((unsigned int)(m >> 4) << 24);
}
// First half of a cluster barrier that orders nothing: the barriers' initialisation has a fence of its own, and what was read of the query block's place is in tensor memory.
// (The releasing form waits for all memory operations of the thread: 1500 clocks ahead of a stream's first tile.)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
template <int REGS> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }
#define PG_REGS_SOFTMAX 144
#define PG_REGS_CONVERT 64
#define PG_REGS_ISSUE 64
static_assert(2 * PG_REGS_SOFTMAX + 2 * PG_REGS_CONVERT + PG_REGS_ISSUE <= 5 * PG_REGS, "the warpgroups' registers come out of the launch's");

template <int ROWS>
__global__ void __launch_bounds__(PG_THREADS, 1)
tree_attn_paged_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ CUtensorMap tmK) {
    using Y = Layout<ROWS>;
    constexpr bool WIDE = ROWS == 256;
    constexpr int REP = ROWS < PG_BM ? PG_BM / ROWS : 1;    // copies of the rows in the 128 lanes
    constexpr int COLS = PG_BN / REP;                      // columns of a tile that a thread takes
    extern __shared__ unsigned char smem_raw[];
    __shared__ int s_seq;
    __shared__ unsigned int s_tmem, s_odd[4];                       // s_odd: tree keys whose value stays out of the product somewhere
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned int base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* gen = smem_raw + (base - smem_u32(smem_raw));
    int* const err = p.c.err;
    // Barriers.  A parity wait tells the current phase from the one before: the next completion of a barrier has to depend on every thread that waits for this one
    // (a unit's and a slot's come round only after it has been handed back, a stream's alternate with its tiles), and the last one has to lie behind it.
    const unsigned int bar_k = base + Y::bar, bar_ek = bar_k + 8 * PG_KEYS, bar_u = bar_ek + 8 * PG_KEYS, bar_eu = bar_u + 8 * Y::units, bar_v = bar_eu + 8 * Y::units,
                       bar_ev = bar_v + 8 * PG_GROUPS, bar_x = bar_ev + 8 * PG_GROUPS, bar_s = bar_x + 8 * PG_EXPS, bar_p = bar_s + 16, bar_sr = bar_p + 16, bar_o = bar_sr + 16,
                       bar_r = bar_o + 16, bar_done = bar_r + 8;
    if (warp == 0) {
        tmem_alloc(smem_u32(&s_tmem), PG_TMEM_COLS);
        tmem_relinquish();
    }
    if (tid < 4) s_odd[tid] = 0u;
    if (tid == 32) {
        for (int i = 0; i < PG_KEYS; ++i) {                  // keys there, S issued
            mbar_init(bar_k + 8 * i, 1);
            mbar_init(bar_ek + 8 * i, 1);
        }
        for (int i = 0; i < Y::units; ++i) {                 // a unit of values there, read
            mbar_init(bar_u + 8 * i, 1);
            mbar_init(bar_eu + 8 * i, PG_CV_THREADS);
        }
        for (int i = 0; i < PG_GROUPS; ++i) {                // a tile of values there, P V issued
            mbar_init(bar_v + 8 * i, PG_CV_THREADS);
            mbar_init(bar_ev + 8 * i, 1);
        }
        for (int i = 0; i < PG_EXPS; ++i) mbar_init(bar_x + 8 * i, PG_CV_THREADS);     // a tile's scales
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s + 8 * i, 1);
            mbar_init(bar_o + 8 * i, 1);
        }
        mbar_init(bar_r, 1);
        mbar_init(bar_done, 1);
    }
    pdl_launch_dependents();
    pdl_wait();
    // Sequences longest first, so that a ragged batch ends on short ones: slot z / hkv is the sequence of that rank by (length descending, index ascending).  More sequences than
    // the block has threads go in their own order.
    int b = blockIdx.z / p.c.hkv;
    const int h = blockIdx.z % p.c.hkv;
    if (p.c.batch > 1 && p.c.batch <= PG_THREADS) {
        if (tid < p.c.batch) {
            const int len = p.c.len[tid];
            int rank = 0;
            for (int j = 0; j < p.c.batch; ++j) {
                const int lj = p.c.len[j];
                rank += (lj > len || (lj == len && j < tid));
            }
            if (rank == b) s_seq = tid;
        }
        __syncthreads();
        b = s_seq;
    }
    const int split = blockIdx.y, ns = p.nsplit, m0 = blockIdx.x * ROWS;
    // the sequence's entries in one round trip
    const int nk_b = p.n_keep[b], st_b = p.status[b], koff = p.keep_off[b], L = kv_length(p.c, b);
    const int nbase = p.layout == HS_ROWS_ORIGINAL ? p.node_off[b] : koff, nend = p.layout == HS_ROWS_ORIGINAL ? p.node_off[b + 1] : koff + nk_b;
    // a tree that passes what the caller stated is left out
    const bool fits = nk_b <= p.max_nodes && nbase >= 0 && nend <= p.max_rows;
    if (st_b == 0 && !fits && tid == 0) atomicCAS(p.c.err, 0, (int)HS_ERR_SHAPE);
    const int nk = st_b == 0 && fits ? max(nk_b, 0) : 0;
    const int M = nk * p.G;
    const bool nothing = m0 >= M;                          // the same for every CTA of the cluster
    // threads of a stream whose warp has a row
    const int active0 = REP > 1 ? PG_BM : min(PG_BM, max(M - m0 + 31, 0) & ~31), active1 = WIDE ? min(PG_BM, max(M - m0 - PG_BM + 31, 0) & ~31) : active0;
    const int tree_tiles = (nk + PG_BN - 1) / PG_BN, tiles = tree_tiles + (L + PG_BN - 1) / PG_BN;
    const int per = (tiles + ns - 1) / ns, g0 = min(split * per, tiles), ntiles = min(per, tiles - g0);
    const int nt = min(max(tree_tiles - g0, 0), ntiles);    // tree tiles of this CTA: its first
    const int live = min(ROWS, M - m0);                  // rows of this block
    const int r_lo = (split * live + ns - 1) / ns, r_hi = ((split + 1) * live + ns - 1) / ns;     // those this CTA merges
    if (tid == 32 && !nothing) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_p + 8 * i, max(i ? active1 : active0, 1));
            mbar_init(bar_sr + 8 * i, max(i ? active1 : active0, 1));
        }
        if (ns > 1) mbar_expect_tx(bar_r, (unsigned int)(ns * (r_hi - r_lo) * PG_ROW_STRIDE));
        mbar_init_fence();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const unsigned int tmem = s_tmem;
    if (nothing) {
        if (warp == 0) tmem_dealloc(tmem, PG_TMEM_COLS);
        return;
    }
    const unsigned int tS = tmem, tO = tmem + 128, tP = tmem + 384, tQ = tmem + 448;
    auto kept_row_of = [&](int node) { return nbase + (p.layout == HS_ROWS_ORIGINAL ? p.keep_idx[koff + node] : node); };
    const int warp_u = __shfl_sync(HS_FULL_MASK, warp, 0);
    float2* s_B = reinterpret_cast<float2*>(gen + Y::exps);             // {B, 2^-B} of tile i at i % PG_EXPS
    float* s_ks = reinterpret_cast<float*>(gen + Y::ks);                // its keys' scales
    unsigned short* s_vs = reinterpret_cast<unsigned short*>(gen + Y::vs);   // its tokens' exponents, as bf16 (integers take the exponential's unit to convert)
    auto exponent_bits = [](unsigned int scale) { return (unsigned short)(__float_as_uint((float)((int)scale - 127)) >> 16); };
    unsigned int* s_red = reinterpret_cast<unsigned int*>(gen + Y::red);

    // A row of 128 bf16 in two halves of a tile becomes its two terms, 128 bytes each, in their place, by the sixteen lanes that brought it, and 2^e in out[]: NaN where
    // something is not finite, which makes NaN of every score it touches.  Rows first, first + 16, ... (four at most) of those below `rows`: their loads and sums go side by side.
    // One row at a time in blocks of few rows, where what counts is how little code is fetched (a token behind 512 7.7 us when this was chosen, with four rows side by side, here and below, 8.8); four above
    // (a tree of 60 behind 100 tokens 11.5, with one 12.0).
    constexpr int TERM_ROWS = REP > 1 ? 1 : 4;
    const int sub = tid & 15;
    // also: scale bytes of other rows, two by two, of which the sixteen lanes find the largest on the way.
    auto to_terms = [&](unsigned char* tile, int half_bytes, int first, int rows, float* out, auto&... also) {
        uint4 w[TERM_ROWS];
        unsigned int a[TERM_ROWS];
#pragma unroll
        for (int j = 0; j < TERM_ROWS; ++j) {
            const int row = first + 16 * j;
            w[j] = row < rows ? *reinterpret_cast<const uint4*>(tile + (sub >> 3) * half_bytes + row * 128 + (((sub & 7) ^ (row & 7)) << 4)) : make_uint4(0u, 0u, 0u, 0u);
            a[j] = max(max(pair_amax(w[j].x), pair_amax(w[j].y)), max(pair_amax(w[j].z), pair_amax(w[j].w)));
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
            for (int j = 0; j < TERM_ROWS; ++j) a[j] = max(a[j], __shfl_xor_sync(HS_FULL_MASK, a[j], o));
            ((also = pair_max(also, __shfl_xor_sync(HS_FULL_MASK, also, o))), ...);
        }                                                // (and every lane has read its part of the rows)
#pragma unroll
        for (int j = 0; j < TERM_ROWS; ++j) {
            const int row = first + 16 * j;
            if (row >= rows) break;                      // (the same for the whole warp: rows is a multiple of 16)
            const int e = a[j] >= 0x7f800000u ? 0 : max((int)((a[j] + 0x1fffffu) >> 23) - 127 - 8, -60);     // the row's largest is at most 1.75 * 2^8
            const unsigned int two = (unsigned int)(127 - e) * 0x00800080u;
            unsigned int t1[4], t2[4];
            e4m3_terms(w[j].x, two, t1[0], t2[0]); e4m3_terms(w[j].y, two, t1[1], t2[1]);
            e4m3_terms(w[j].z, two, t1[2], t2[2]); e4m3_terms(w[j].w, two, t1[3], t2[3]);
            unsigned char* at = tile + row * 128 + (((sub >> 1) ^ (row & 7)) << 4) + (sub & 1) * 8;
            *reinterpret_cast<uint2*>(at) = make_uint2(e4m3_bytes(t1[0], t1[1]), e4m3_bytes(t1[2], t1[3]));
            *reinterpret_cast<uint2*>(at + half_bytes) = make_uint2(e4m3_bytes(t2[0], t2[1]), e4m3_bytes(t2[2], t2[3]));
            if (sub == 0) out[row] = a[j] >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : power_of_two(e);
        }
    };

    if (warp_u >= 8) {
        if (warp_u < 16) give_registers<PG_REGS_CONVERT>();
        else give_registers<PG_REGS_ISSUE>();
        // First half of a cluster barrier (128 rows): when it completes every CTA of the cluster has its barriers and is through with the query block, and
        // that place may be written from outside.
        if (!WIDE && ns > 1) cluster_arrive_relaxed();
        const int ct8 = tid - PG_SM_THREADS;                 // (of the converters' 256)
        if (warp_u < 16) {
#pragma unroll 1
            for (int j = ct8 >> 4; j < nt * PG_BN; j += 16) {
                const int key = g0 * PG_BN + j;
                const bool there = key < nk;
                const size_t from = (there ? (size_t)kept_row_of(key) * p.c.hkv + h : 0) * HS_HEAD_DIM + sub * 8;
                const unsigned int to = (j >> 6) * PG_TILE_BYTES + pg_off(PG_BN, j & (PG_BN - 1), sub);
                copy16(base + Y::k + to, p.k_tree + from, there);
                copy16(base + Y::v + to, p.v_tree + from, there);
            }
        }
        // Until the query and tree rows are asked for nobody asks for the prefix (behind eight units they would come late) or polls a barrier (which takes issue slots), and the
        // issuers sleep until the queries are in tensor memory.
        if (warp_u == PG_WARP_S || warp_u == PG_WARP_PV) named_bar_sync(3, PG_SM_THREADS + 64);
        else named_bar_sync(2, PG_THREADS - 64);
        // The prefix tiles' pages.  A copy is issued by one lane while all run its loop, so that addresses stay uniform; it takes a warp 150 clocks all the same, and a tile of
        // 32-token pages eight of them: two warps ask for keys, and every group of converters for its own values and scales.
        const int t_first = (g0 + nt - tree_tiles) * PG_BN;                  // first token of this CTA's prefix tiles
        const int lg = p.c.log_page, page = 1 << lg, run = min(page, PG_BN), per_tile = PG_BN / run;
        const int* table = p.c.table + (size_t)b * p.c.max_pages;
        const int last_page = (L - 1) >> lg;
        // lane k: entry of page k of the tile that starts at tok, where there is one (pages behind the last token are not read)
        auto entry_of = [&](int tok) { const int i = (tok >> lg) + lane; return lane < per_tile && i <= last_page ? table[i] : 0; };
        auto pieces_of = [&](int tok) { return min(per_tile, (min(L - tok, PG_BN) + run - 1) / run); };
        // row (of 128 bytes, and of the scales) of piece k of a tile
        auto row_of = [&](int entry, int tok, int k) {
            int id = __shfl_sync(HS_FULL_MASK, entry, k);
            if ((unsigned int)id >= (unsigned int)p.c.n_pages) {
                if (lane == 0) kv_bad_page(err);
                id = 0;
            }
            return (((size_t)(unsigned int)id * p.c.hkv + h) << lg) + (tok & (page - 1));      // (pages below 64 tokens: a tile starts on one)
        };
        if (warp_u < 16) {
            // ---- the converters: four groups of two warps, each the values of every fourth prefix tile.  (A round is a chain of waits, loads, the tile's exponent and the
            // stores, most of it latency.) -----------------------------------------------------------------------------------------------------------
            const int group = (warp_u - 8) >> 1, ct = tid & (PG_CV_THREADS - 1);
            // A thread has a key's bytes, eight chunks of 16, and takes them in the order c ^ key, so that neither the loads nor the stores of eight lanes use a bank
            // twice: chunk j lies at 16 j of its row, its two chunks of f16 values in half j >> 2 of the tile at 2 j & 7, swizzled by the key.
            const int key = ct, turn = key & 7, slot = (nt + group) & (PG_GROUPS - 1);
            unsigned int load_at[4], even_at[4], odd_at[4];          // of chunks c ^ turn, c = 0 .. 3; those of c = 4 .. 7 lie at fixed distances
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = c ^ turn;
                load_at[c] = key * HS_HEAD_DIM + j * 16;
                even_at[c] = (j >> 2) * (PG_TILE_BYTES / 2) + key * 128 + (((2 * j) & 7) ^ turn) * 16;
                odd_at[c] = even_at[c] ^ 16u;
            }
            const int load_on = turn < 4 ? 64 : -64, store_on = turn < 4 ? PG_TILE_BYTES / 2 : -(PG_TILE_BYTES / 2);
            unsigned char* to = gen + Y::v + slot * PG_TILE_BYTES;
            // A unit of values (by the group's first warp) and its scale bytes (by the other).
            auto ask = [&](int entry, int tok, int unit) {
                const int pieces = pieces_of(tok);
                const unsigned int bar = bar_u + unit * 8;
                const bool scale_warp = warp_u & 1;
                if (!scale_warp && elect_one()) mbar_expect_tx(bar, (unsigned int)(pieces * run * (HS_HEAD_DIM + 2)));
                __syncwarp();
#pragma unroll 1
                for (int k = 0; k < pieces; ++k) {
                    const size_t src = row_of(entry, tok, k);
                    if (elect_one()) {
                        if (scale_warp) {
                            const unsigned int at = base + Y::scale + unit * 2 * PG_BN + k * run;
                            bulk_load(at, p.c.v_scale + src, run, bar);
                            bulk_load(at + PG_BN, p.c.k_scale + src, run, bar);
                        } else {
                            bulk_load(base + Y::unit + unit * PG_UNIT_BYTES + k * run * HS_HEAD_DIM, p.c.v + src * HS_HEAD_DIM, run * HS_HEAD_DIM, bar);
                        }
                    }
                    __syncwarp();
                }
            };
            for (int u = group; u < Y::units && nt + u < ntiles; u += PG_GROUPS) {
                const int tok = t_first + u * PG_BN;
                ask(entry_of(tok), tok, u);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();                                    // (rows are read by other lanes than those that brought them)
            // The tree's tiles: keys as terms; values as f16 relative to their exponents, without those that stay apart.
#pragma unroll 1
            for (int t = 0; t < nt; ++t) {
                unsigned char* tile = gen + Y::v + t * PG_TILE_BYTES;
                unsigned int hi = 0u, lo = 255u;             // of the live tokens' scale bytes
                const int live_keys = nk - (g0 + t) * PG_BN, keys16 = min(PG_BN, (live_keys + 15) & ~15);       // (those behind them are masked, and zeros)
                [[maybe_unused]] uint4 v[PG_BN / 16];
                [[maybe_unused]] unsigned int pair[PG_BN / 32];              // scale bytes of two rows
                auto scale_of = [&](int j) { return pair[j >> 1] >> (j & 1) * 16 & 255u; };
                if constexpr (REP > 1) {                     // a row at a time, read again below
                    if (ct8 >= keys16 && ct8 < PG_BN) s_vs[t * PG_BN + ct8] = 0;     // (masked, but no number would reach the row's sum)
#pragma unroll 1
                    for (int row = ct8 >> 4; row < keys16; row += 16) {
                        uint4* at = reinterpret_cast<uint4*>(tile + pg_off(PG_BN, row, sub));
                        uint4 x = *at;
                        unsigned int m = max(max(pair_amax(x.x), pair_amax(x.y)), max(pair_amax(x.z), pair_amax(x.w)));
                        if (m >= PG_APART) {
                            x = make_uint4(near_or_zero(x.x), near_or_zero(x.y), near_or_zero(x.z), near_or_zero(x.w));
                            m = PG_APART;
                            *at = x;
                            const int key = (g0 + t) * PG_BN + row;
                            atomicOr(&s_odd[key >> 5], 1u << (key & 31));
                        }
                        __syncwarp();
                        unsigned int scale = e8m0_of(m);
                        to_terms(gen + Y::k + t * 2 * PG_UNIT_BYTES, PG_UNIT_BYTES, row, keys16, s_ks + t * PG_BN, scale);
                        scale = max(scale, PG_SMALLEST);
                        if (sub == 0) s_vs[t * PG_BN + row] = exponent_bits(scale);
                        if (row < live_keys) {
                            hi = max(hi, scale);
                            lo = min(lo, scale);
                        }
                    }
                } else {
                    to_terms(gen + Y::k + t * 2 * PG_UNIT_BYTES, PG_UNIT_BYTES, ct8 >> 4, keys16, s_ks + t * PG_BN);
                    unsigned int behind[PG_BN / 32];                             // 255 in the place of rows behind the last
#pragma unroll
                    for (int j = 0; j < PG_BN / 16; ++j) {
                        const int row = (ct8 >> 4) + 16 * j;
                        v[j] = row < keys16 ? *reinterpret_cast<const uint4*>(tile + pg_off(PG_BN, row, sub)) : make_uint4(0u, 0u, 0u, 0u);
                        unsigned int m = max(max(pair_amax(v[j].x), pair_amax(v[j].y)), max(pair_amax(v[j].z), pair_amax(v[j].w)));
                        if (m >= PG_APART) {
                            v[j] = make_uint4(near_or_zero(v[j].x), near_or_zero(v[j].y), near_or_zero(v[j].z), near_or_zero(v[j].w));
                            m = PG_APART;
                            const int key = (g0 + t) * PG_BN + row;
                            atomicOr(&s_odd[key >> 5], 1u << (key & 31));
                        }
                        const unsigned int none = row < live_keys ? 0u : 255u;
                        pair[j >> 1] = j & 1 ? pair[j >> 1] | e8m0_of(m) << 16 : e8m0_of(m);
                        behind[j >> 1] = j & 1 ? behind[j >> 1] | none << 16 : none;
                    }
                    __syncwarp();
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
                        for (int j = 0; j < PG_BN / 32; ++j) pair[j] = pair_max(pair[j], __shfl_xor_sync(HS_FULL_MASK, pair[j], o));
                    }
                    unsigned int h2 = 0u, l2 = 0x00ff00ffu;
#pragma unroll
                    for (int j = 0; j < PG_BN / 32; ++j) {
                        pair[j] = pair_max(pair[j], PG_SMALLEST * 0x10001u);
                        h2 = pair_max(h2, pair[j]);                              // (rows behind the last are the smallest)
                        l2 = pair_min(l2, pair[j] | behind[j]);
                    }
                    hi = max(h2 & 255u, h2 >> 16);
                    lo = min(l2 & 255u, l2 >> 16);
                }
                hi = __reduce_max_sync(HS_FULL_MASK, hi);
                lo = __reduce_min_sync(HS_FULL_MASK, lo);
                if (lane < 2) s_red[warp - 8 + 8 * lane] = lane ? lo : hi;
                named_bar_sync(4, PG_SM_THREADS);
                const unsigned int red = s_red[lane & 15];
                hi = __reduce_max_sync(HS_FULL_MASK, lane & 8 ? 0u : red);
                lo = __reduce_min_sync(HS_FULL_MASK, lane & 8 ? red : 255u);
                const bool flat = hi <= lo + PG_FLAT;
                if constexpr (REP > 1) {
#pragma unroll 1
                    for (int row = ct8 >> 4; row < keys16; row += 16) {
                        uint4* at = reinterpret_cast<uint4*>(tile + pg_off(PG_BN, row, sub));
                        const uint4 x = *at;
                        const float f = power_of_two(flat ? 127 - (int)hi : -(int)__uint_as_float((unsigned int)s_vs[t * PG_BN + row] << 16));
                        *at = make_uint4(scaled_half2(x.x, f), scaled_half2(x.y, f), scaled_half2(x.z, f), scaled_half2(x.w, f));
                    }
                } else {
                    if (flat) pair[0] = pair[1] = hi * 0x10001u;
#pragma unroll
                    for (int j = 0; j < PG_BN / 16; ++j) {
                        const int row = (ct8 >> 4) + 16 * j;
                        const float f = power_of_two(127 - (int)scale_of(j));
                        if (!flat && sub == 0) s_vs[t * PG_BN + row] = exponent_bits(scale_of(j));
                        if (row < keys16)
                            *reinterpret_cast<uint4*>(tile + pg_off(PG_BN, row, sub)) = make_uint4(scaled_half2(v[j].x, f), scaled_half2(v[j].y, f), scaled_half2(v[j].z, f), scaled_half2(v[j].w, f));
                    }
                }
                if (ct8 == 0) s_B[t] = flat ? make_float2((float)((int)hi - 127), power_of_two(127 - (int)hi)) : make_float2(0.f, 0.f);
                fence_proxy_async_smem();
                named_bar_sync(4, PG_SM_THREADS);
                // what the loader and a group would bring to the tile's barriers
                if (ct8 < PG_CV_THREADS) {
                    mbar_arrive(bar_x + t * 8);
                    mbar_arrive(bar_v + t * 8);
                }
                if (ct8 < 2) mbar_arrive(bar_k + (2 * t + ct8) * 8);
            }
            unsigned int phase = 0u;
            int unit = group;
            bool ok = false;                                 // the next unit is there
#pragma unroll 1
            for (int i = nt + group; i < ntiles; i += PG_GROUPS) {
                const unsigned char* from = gen + Y::unit + unit * PG_UNIT_BYTES;
                const unsigned char* scales = gen + Y::scale + unit * 2 * PG_BN;
                const int left = L - (g0 + i - tree_tiles) * PG_BN;  // keys of the tile inside the sequence
                const int next_tok = t_first + (i - nt + Y::units) * PG_BN;  // of the tile that this unit takes next
                const int next_entry = entry_of(next_tok);
                if (!ok) mbar_wait(bar_u + unit * 8, phase, err);
                __syncwarp();
                const unsigned int two = *reinterpret_cast<const unsigned short*>(scales + 2 * lane), s_key = scales[PG_BN + key];
                const int s = scales[key];
                uint4 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = *reinterpret_cast<const uint4*>(from + load_at[c]);
                const unsigned int back_phase = ((unsigned int)(i / PG_GROUPS) & 1u) ^ 1u;
                bool back = true;                            // the tile's place is free
                if (i >= PG_GROUPS) back = mbar_test_wait(bar_ev + slot * 8, back_phase);
                const unsigned int sa = two & 255u, sb = two >> 8;
                const bool la = 2 * lane < left && sa != 255u, lb = 2 * lane + 1 < left && sb != 255u;      // (a token of no number has no size)
                const int hi = token_exponent(__reduce_max_sync(HS_FULL_MASK, max(la ? sa : 0u, lb ? sb : 0u)));
                const int lo = token_exponent(__reduce_min_sync(HS_FULL_MASK, min(la ? sa : 255u, lb ? sb : 255u)));
                const bool flat = hi - lo <= PG_FLAT;
                const int e = flat ? hi : token_exponent(s);
                // The tile's scales, ahead of S.  (Their places were last used eight tiles back, by a P V that this group has waited for.)  A row of scale byte 255 is NaN
                // whatever its bytes are.
                s_ks[(i & (PG_EXPS - 1)) * PG_BN + key] = __uint_as_float(s_key == 255u ? 0x7fffffffu : s_key << 23);
                if (ct == 0) s_B[i & (PG_EXPS - 1)] = flat ? make_float2((float)hi, power_of_two(-hi)) : make_float2(0.f, 0.f);
                if (!flat) s_vs[(i & (PG_EXPS - 1)) * PG_BN + key] = exponent_bits((unsigned int)(e + 127));
                mbar_arrive(bar_x + (i & (PG_EXPS - 1)) * 8);
                // (behind the last key the factor is zero: spread bytes are finite, whatever they were)
                const unsigned int f = key >= left ? 0u : s == 255 ? 0x7fff7fffu : half2_power(s - 127 - e + 8);
                if (!back) mbar_wait(bar_ev + slot * 8, back_phase, err);
                const unsigned char* src = from + load_on;
                unsigned char* dst = to;
#pragma unroll 1                                             // (code that runs a few times in a short call is paid for when it is fetched)
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint2 o0 = e4m3_half4(w[c].x, f), o1 = e4m3_half4(w[c].y, f), o2 = e4m3_half4(w[c].z, f), o3 = e4m3_half4(w[c].w, f);
                        *reinterpret_cast<uint4*>(dst + even_at[c]) = make_uint4(o0.x, o0.y, o1.x, o1.y);
                        *reinterpret_cast<uint4*>(dst + odd_at[c]) = make_uint4(o2.x, o2.y, o3.x, o3.y);
                        if (half == 0) w[c] = *reinterpret_cast<const uint4*>(src + load_at[c]);
                    }
                    dst += store_on;
                }
                mbar_arrive(bar_eu + unit * 8);
                fence_proxy_async_smem();
                mbar_arrive(bar_v + slot * 8);
                if (i + Y::units < ntiles) {
                    mbar_wait(bar_eu + unit * 8, phase, err);        // both warps have read the unit
                    __syncwarp();
                    ask(next_entry, next_tok, unit);
                }
                phase ^= unit + PG_GROUPS < Y::units ? 0u : 1u;
                unit = unit + PG_GROUPS < Y::units ? unit + PG_GROUPS : group;
                ok = mbar_test_wait(bar_u + unit * 8, phase);
            }
        } else if (warp_u == PG_WARP_S) {
            // ---- S = Q K^T of tile i as soon as K and the scales are there and the stream has its last S in registers -------------------------
            const unsigned int idesc = umma_idesc_e4m3(PG_BM, PG_BN);
            const unsigned long long dk0 = umma_desc_sw128(base + Y::k, 16, 1024);
            const unsigned long long dq1 = umma_desc_sw128(base + Y::q + PG_BM * HS_HEAD_DIM * 2, 16, 1024);      // the second block of 256 rows
            tc_fence_after_sync();                           // Q is in tensor memory
            unsigned int phase = 0u;
            int at = 0;                                      // place of the next keys
            // S of stream g (+)= Q K^T for the keys at a place
            auto product = [&](int g, int place, bool more) {
                const unsigned long long dk = dk0 + (unsigned long long)(place * (PG_UNIT_BYTES >> 4));
                const unsigned int to = tS + g * PG_BN;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    if (WIDE && g == 1) umma_ss_e4m3(to, dq1 + (((ks >> 2) * (PG_BM * 128) + (ks & 3) * 32) >> 4), dk + ((ks & 3) * 32 >> 4), idesc, more || ks > 0 ? 1u : 0u);
                    else umma_ts_e4m3(to, tQ + ks * 8, dk + ((ks & 3) * 32 >> 4), idesc, more || ks > 0 ? 1u : 0u);
                }
            };
#pragma unroll 1
            for (int i = 0; i < nt; ++i) {                   // tree tiles: both terms of their keys, side by side
                mbar_wait(bar_k + 2 * i * 8, 0u, err);
                mbar_wait(bar_k + (2 * i + 1) * 8, 0u, err);
                mbar_wait(bar_x + i * 8, 0u, err);
#pragma unroll
                for (int g = 0; g < (WIDE ? 2 : 1); ++g) {
                    if (WIDE && g == 1 && active1 == 0) continue;
                    if (WIDE && i == 1) mbar_wait(bar_sr + g * 8, 0u, err);
                    __syncwarp();
                    tc_fence_after_sync();
                    if (elect_one()) {
#pragma unroll 1
                        for (int k = 0; k < 2; ++k) product(WIDE ? g : i, 2 * i + k, k == 1);
                        umma_commit(bar_s + (WIDE ? g : i) * 8);
                        if (!WIDE || g == 1 || active1 == 0) {
                            umma_commit(bar_ek + 2 * i * 8);
                            umma_commit(bar_ek + (2 * i + 1) * 8);
                        }
                    }
                    __syncwarp();
                }
            }
            at = 2 * nt;
#pragma unroll 1
            for (int i = nt; i < ntiles; ++i) {
                const unsigned int bar_x_i = bar_x + (i & (PG_EXPS - 1)) * 8, x_phase = (unsigned int)(i / PG_EXPS) & 1u;
                // (asked together: an answer takes 123 clocks)
                const bool ok_k = mbar_test_wait(bar_k + at * 8, phase), ok_x = mbar_test_wait(bar_x_i, x_phase);
                const unsigned int sr_bar = bar_sr + (WIDE ? 0 : (i & 1) * 8), sr_phase = WIDE ? (unsigned int)(i - 1) & 1u : (unsigned int)((i >> 1) - 1) & 1u;
                const bool ok_r = i < (WIDE ? 1 : 2) || mbar_test_wait(sr_bar, sr_phase);
                if (!ok_k) mbar_wait(bar_k + at * 8, phase, err);
                if (!ok_x) mbar_wait(bar_x_i, x_phase, err);
                if (!ok_r) mbar_wait(sr_bar, sr_phase, err);
                __syncwarp();
                tc_fence_after_sync();
                if (elect_one()) {
                    product(WIDE ? 0 : (i & 1), at, false);
                    umma_commit(bar_s + (WIDE ? 0 : (i & 1) * 8));
                    if (!WIDE || active1 == 0) umma_commit(bar_ek + at * 8);
                }
                __syncwarp();
                if (WIDE && active1 > 0) {
                    if (i >= 1) mbar_wait(bar_sr + 8, (unsigned int)(i - 1) & 1u, err);
                    __syncwarp();
                    tc_fence_after_sync();
                    if (elect_one()) {
                        product(1, at, false);
                        umma_commit(bar_s + 8);
                        umma_commit(bar_ek + at * 8);
                    }
                    __syncwarp();
                }
                phase ^= at == PG_KEYS - 1 ? 1u : 0u;
                at = at == PG_KEYS - 1 ? 0 : at + 1;
            }
        } else if (warp_u == PG_WARP_PV) {
            // ---- O += P V of the streams' tiles ----------------------------------------------------------------------------------------
            const unsigned int idesc = umma_idesc_half(PG_BM, HS_HEAD_DIM, true);
            const unsigned long long dv0 = umma_desc_sw128(base + Y::v, PG_TILE_BYTES / 2, 1024);
#pragma unroll 1
            for (int i = 0; i < ntiles; ++i) {
                const int slot = i & (PG_GROUPS - 1);
                const unsigned long long dv = dv0 + (unsigned long long)(slot * (PG_TILE_BYTES >> 4));
                mbar_wait(bar_v + slot * 8, (unsigned int)(i / PG_GROUPS) & 1u, err);
#pragma unroll
                for (int k = 0; k < (WIDE ? 2 : 1); ++k) {
                    const int g = WIDE ? k : i & 1, n = WIDE ? i : i >> 1;      // stream, and its tile's number
                    const bool last = !WIDE || k == 1 || active1 == 0;
                    if (WIDE && k == 1 && active1 == 0) continue;
                    mbar_wait(bar_p + g * 8, (unsigned int)n & 1u, err);
                    __syncwarp();
                    tc_fence_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            umma_ts_bf16(tO + g * HS_HEAD_DIM, tP + g * (PG_BN / 2) + kk * 8, dv + (kk * 2048 >> 4), idesc, (n > 0 || kk > 0) ? 1u : 0u);
                        umma_commit(bar_o + g * 8);
                        if (last) umma_commit(bar_ev + slot * 8);
                        if (last && i == ntiles - 1) umma_commit(bar_done);     // every S was read before the last P was written: all products are complete
                    }
                    __syncwarp();
                }
            }
        } else {
            // ---- the loaders of keys, of the even and of the odd prefix tiles ---------------------------------------------------------------------------
            const int odd = warp_u - PG_WARP_LOAD;
            int place = 2 * nt + odd >= PG_KEYS ? 2 * nt + odd - PG_KEYS : 2 * nt + odd;      // (the tree's terms have the first places)
            int used = 2 * nt + odd;
            unsigned int phase = used >= PG_KEYS ? 1u : 0u;
            int entry = nt + odd < ntiles ? entry_of(t_first + odd * PG_BN) : 0;
#pragma unroll 1
            for (int i = nt + odd; i < ntiles; i += 2) {
                const int tok = t_first + (i - nt) * PG_BN, pieces = pieces_of(tok);
                const int next_entry = entry_of(tok + 2 * PG_BN);
                const unsigned int bar = bar_k + place * 8;
                if (used >= PG_KEYS) mbar_wait(bar_ek + place * 8, phase ^ 1u, err);
                __syncwarp();
                if (elect_one()) mbar_expect_tx(bar, (unsigned int)(pieces * run * HS_HEAD_DIM));
                __syncwarp();
#pragma unroll 1
                for (int k = 0; k < pieces; ++k) {
                    const size_t src = row_of(entry, tok, k);
                    if (elect_one()) tma_load_2d(base + Y::k + place * PG_UNIT_BYTES + k * run * HS_HEAD_DIM, &tmK, 0, (int)src, bar);
                    __syncwarp();
                }
                entry = next_entry;
                used += 2;
                phase ^= place + 2 < PG_KEYS ? 0u : 1u;
                place = place + 2 < PG_KEYS ? place + 2 : place + 2 - PG_KEYS;
            }
        }
        __syncwarp();
        if (ns > 1) {
            if (WIDE) cluster_arrive();
            cluster_wait();
        }
        return;
    }

    // ---- the softmax warps -----------------------------------------------------------------------------------------------------------------
    take_registers<PG_REGS_SOFTMAX>();
    const unsigned int lane_off = (unsigned int)((warp & 3) * 32) << 16;       // a warp reaches lanes 32 * (warp % 4) ..
    const int lane_row = tid & (PG_BM - 1), half = tid >> 7;                    // the thread's lane of tensor memory, and its stream
    const int row = REP > 1 ? lane_row % ROWS : lane_row, copy = REP > 1 ? lane_row / ROWS : 0;      // its query row in the block, and which of the row's copies
    const bool act = (lane_row & ~31) < (half ? active1 : active0);
    // Query rows into shared memory, 16 lanes a row, asked for at once and ahead of the prefix's; rows past the last are zero.  In rolled loops: what runs once costs 12 clocks
    // an instruction, for its fetching (the same loads through registers, unrolled, took 5000 clocks).  The converters do the same with the tree's tiles meanwhile.
    float* s_qs = reinterpret_cast<float*>(gen + Y::qs);
    {
        const int rows16 = min(ROWS, (live + 15) & ~15);     // (rows of the block beyond them stay as they are: nobody looks at what becomes of them)
#pragma unroll 1
        for (int at = tid >> 4; at < rows16; at += 16) {
            const int rr = m0 + at, node = (int)((unsigned int)rr * p.inv_g >> 16);
            const bool there = at < live;
            const size_t from = there ? (size_t)kept_row_of(node) * p.hq + h * p.G + (rr - node * p.G) : 0;
            copy16(base + Y::q + (at >> 7) * (PG_BM * HS_HEAD_DIM * 2) + pg_off(PG_BM, at & (PG_BM - 1), sub), p.q + from * HS_HEAD_DIM + sub * 8, there);
        }
        asm volatile("bar.arrive 2, %0;" ::"r"(PG_THREADS - 64) : "memory");
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();                                        // (rows are read by other lanes than those that brought them)
#pragma unroll 1
        for (int at = 0; at < rows16; at += 16 * TERM_ROWS) {
            const int in_block = at & (PG_BM - 1);
            to_terms(gen + Y::q + (at >> 7) * (PG_BM * HS_HEAD_DIM * 2), PG_BM * 128, in_block + (tid >> 4), in_block + rows16 - at, s_qs + at - in_block);
        }
    }
    // this thread's own row: its ancestor mask and output row
    const int r = m0 + (WIDE ? half * PG_BM : 0) + row;
    long long orow = -1;
    unsigned long long mk0 = 0ull, mk1 = 0ull;
    if (r < M) {
        const int node = (int)((unsigned int)r * p.inv_g >> 16);
        orow = (long long)kept_row_of(node) * p.hq + h * p.G + (r - node * p.G);
        mk0 = p.anc_mask[2 * (size_t)(koff + node)];
        mk1 = p.anc_mask[2 * (size_t)(koff + node) + 1];
    }
    if (WIDE) fence_proxy_async_smem();                      // (the second block is read by the tensor cores)
    named_bar_sync(1, PG_SM_THREADS);
    float row_scale = p.scale_log2 * s_qs[(WIDE ? half * PG_BM : 0) + row];
    if (row_scale < 1e-35f) row_scale = 1e-35f;              // (0 * -inf in a masked column would be NaN, and a token's exponent over it stays finite; a NaN stays)
    if (!WIDE || half == 0) {
#pragma unroll 1
        for (int c0 = WIDE ? 0 : half * 8; c0 < (WIDE ? 16 : half * 8 + 8); c0 += 4) {
            uint4 qv[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) qv[c] = *reinterpret_cast<const uint4*>(gen + Y::q + pg_off(PG_BM, row, c0 + c));
            tmem_st16(tQ + c0 * 4 + lane_off, reinterpret_cast<unsigned int*>(qv));
        }
        if (REP > 1) {                                       // P of the columns that other copies take stays zero
            unsigned int zero[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) zero[c] = 0u;
            tmem_st32(tP + half * (PG_BN / 2) + lane_off, zero);
        }
        tmem_wait_st();
    }
    tc_fence_before_sync();
    asm volatile("bar.arrive 3, %0;" ::"r"(PG_SM_THREADS + 64) : "memory");
    __syncwarp();
    if (!WIDE && ns > 1) cluster_arrive_relaxed();

    // The stream's tiles.  As soon as S is in registers its buffer is handed back.  The stream's P buffer and O were last used by its last O += P V, which is
    // waited for before they are touched.  Both barriers are asked ahead of other work: an answer takes 123 clocks.
    float mrun = -CUDART_INF_F, lrun = 0.f, prun = 0.f;      // prun: the sum of P, which bounds O
    {
        unsigned int sr[COLS];
        // The reference of the exponents follows the maximum only when that has grown by more than 8: until then P <= 2^14 instead of <= 2^6, which f16
        // holds as exactly, and O is rescaled a few times per row instead of whenever any row of the warp sees a new maximum.
        auto follow = [&](float mx) { return (mx > mrun + 8.f || mrun == -CUDART_INF_F) ? fmaxf(mrun, mx) : mrun; };
        bool ok_s = false;
        int n = 0;                                           // the stream's tiles so far
#pragma unroll 1
        for (int i = WIDE ? 0 : half; i < ntiles && act; i += WIDE ? 1 : 2, ++n) {
            if (!ok_s) mbar_wait(bar_s + half * 8, (unsigned int)n & 1u, err);
            __syncwarp();
            tc_fence_after_sync();
            const unsigned int s_at = tS + half * PG_BN + copy * COLS + lane_off;
            if constexpr (COLS == 16) {
                tmem_ld16(s_at, sr);
            } else {
                tmem_ld32(s_at, sr);
                if constexpr (COLS == 64) tmem_ld32(s_at + 32, sr + 32);
            }
            const float2 eb = s_B[i & (PG_EXPS - 1)];
            const float4* ks = reinterpret_cast<const float4*>(s_ks + (i & (PG_EXPS - 1)) * PG_BN + copy * COLS);
            tmem_wait_ld();
            tc_fence_before_sync();
            mbar_arrive(bar_sr + half * 8);
            // the keys' scales
#pragma unroll
            for (int c = 0; c < COLS; c += 4) {
                const float4 k4 = ks[c >> 2];
                const float2 a = mul2_ftz(make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), make_float2(k4.x, k4.y));
                const float2 d = mul2_ftz(make_float2(__uint_as_float(sr[c + 2]), __uint_as_float(sr[c + 3])), make_float2(k4.z, k4.w));
                sr[c] = __float_as_uint(a.x); sr[c + 1] = __float_as_uint(a.y); sr[c + 2] = __float_as_uint(d.x); sr[c + 3] = __float_as_uint(d.y);
            }

            const bool is_tree = i < nt;
            const int col0 = (is_tree ? g0 + i : g0 + i - tree_tiles) * PG_BN;
            const int nvis = (is_tree ? nk : L) - col0;
            float sum = 0.f;                                 // of 2^(t - R), where the tile's tokens have exponents of their own
            if (is_tree || nvis < PG_BN || eb.y == 0.f) {    // (one branch for what is rare: a second one in the chain costs every tile, long trees 380 to 393 us)
                unsigned long long vis64 = nvis >= 64 ? ~0ull : ((1ull << max(nvis, 0)) - 1ull);
                if (is_tree) vis64 &= (col0 == 0 ? mk0 : mk1);
                vis64 >>= copy * COLS;
                const unsigned int vlo = (unsigned int)vis64, vhi = (unsigned int)(vis64 >> 32);
#pragma unroll
                for (int c = 0; c < COLS; ++c)
                    if (!(((c < 32 ? vlo : vhi) >> (c & 31)) & 1u)) sr[c] = __float_as_uint(-CUDART_INF_F);
                if (eb.y == 0.f) {                           // t + B in place of t
                    // (volatile: read twice rather than kept, the registers are full)
                    const volatile unsigned int* vs = reinterpret_cast<const volatile unsigned int*>(s_vs + (i & (PG_EXPS - 1)) * PG_BN + copy * COLS);
                    const float inv = rcp_approx(row_scale);
                    float ta = -CUDART_INF_F, tb = -CUDART_INF_F;
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        const unsigned int w = vs[c >> 1];
                        const float2 x = fma2_ftz(make_float2(bf16_lo(w), bf16_hi(w)), make_float2(inv, inv), make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])));
                        sr[c] = __float_as_uint(x.x); sr[c + 1] = __float_as_uint(x.y);
                        ta = fmaxf(ta, x.x); tb = fmaxf(tb, x.y);
                    }
                    const float m = follow(fmaxf(ta, tb) * row_scale), shift = PG_LIFT - (m == -CUDART_INF_F ? 0.f : m);
                    float2 total = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        const unsigned int w = vs[c >> 1];
                        const float2 x = fma2_ftz(make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), make_float2(row_scale, row_scale), make_float2(shift, shift));
                        const float2 y = fma2_ftz(make_float2(bf16_lo(w), bf16_hi(w)), make_float2(-1.f, -1.f), x);
                        total = add2_ftz(total, make_float2(ex2_approx(y.x), ex2_approx(y.y)));
                    }
                    sum = total.x + total.y;
                }
            }
            float mxa = -CUDART_INF_F, mxb = -CUDART_INF_F;
#pragma unroll
            for (int c = 0; c < COLS / 2; c += 2) {
                mxa = max3(mxa, __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
                mxb = max3(mxb, __uint_as_float(sr[COLS / 2 + c]), __uint_as_float(sr[COLS / 2 + c + 1]));
            }
            // (the scale is positive: it commutes with the maximum and folds into the exponent's multiply-add)
            const float mx = fmaf(fmaxf(mxa, mxb), row_scale, eb.x);
            const float mnew = follow(mx), muse = (mnew == -CUDART_INF_F) ? 0.f : mnew;
            const float corr = ex2_approx(mrun - muse);
            mrun = mnew;
            const float2 sc2 = make_float2(row_scale, row_scale), nm2 = make_float2(eb.x - muse + PG_LIFT, eb.x - muse + PG_LIFT);
            float2 ls0 = make_float2(0.f, 0.f), ls1 = make_float2(0.f, 0.f);
            uint4 pk[COLS / 8];
            bool ok_o = false;                               // the stream's last O += P V is complete
#pragma unroll
            for (int c8 = 0; c8 < COLS / 8; ++c8) {
                if (c8 == COLS / 16) ok_o = mbar_test_wait(bar_o + half * 8, (unsigned int)(n + 1) & 1u);
                float2 pv[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 x = fma2_ftz(make_float2(__uint_as_float(sr[c8 * 8 + 2 * e]), __uint_as_float(sr[c8 * 8 + 2 * e + 1])), sc2, nm2);
                    pv[e] = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                }
                ls0 = add2_ftz(ls0, add2_ftz(pv[0], pv[1]));
                ls1 = add2_ftz(ls1, add2_ftz(pv[2], pv[3]));
                // P in f16, off by at most 2^-11 of itself each; the sum keeps the unrounded values
                pk[c8].x = pg_pack_half(pv[0].x, pv[0].y); pk[c8].y = pg_pack_half(pv[1].x, pv[1].y);
                pk[c8].z = pg_pack_half(pv[2].x, pv[2].y); pk[c8].w = pg_pack_half(pv[3].x, pv[3].y);
            }
            const float2 ls = add2_ftz(ls0, ls1);
            prun = fmaf(prun, corr, ls.x + ls.y);
            lrun = fmaf(lrun, corr, fmaf(ls.x + ls.y, eb.y, sum));
            if (n >= 1) {
                if (!ok_o) mbar_wait(bar_o + half * 8, (unsigned int)(n + 1) & 1u, err);
                tc_fence_after_sync();
            }
            // rescale this stream's O (warp-wide; the vote is where the lanes meet again; lanes without a row hold anything)
            if (n >= 1 && __any_sync(HS_FULL_MASK, corr != 1.f && r < M)) {
#pragma unroll 1
                for (int ch = 0; ch < HS_HEAD_DIM; ch += 32) {
                    unsigned int ov[32];
                    const unsigned int at = tO + half * HS_HEAD_DIM + lane_off + ch;
                    tmem_ld32(at, ov);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 32; ++c) ov[c] = __float_as_uint(__uint_as_float(ov[c]) * corr);
                    tmem_st32(at, ov);
                }
            }
            ok_s = mbar_test_wait(bar_s + half * 8, (unsigned int)(n + 1) & 1u);
            __syncwarp();
            const unsigned int p_at = tP + half * (PG_BN / 2) + copy * (COLS / 2) + lane_off;
            if constexpr (COLS == 64) tmem_st32(p_at, reinterpret_cast<unsigned int*>(pk));
            else if constexpr (COLS == 32) tmem_st16(p_at, reinterpret_cast<unsigned int*>(pk));
            else tmem_st8(p_at, reinterpret_cast<unsigned int*>(pk));
            tmem_wait_st();
            tc_fence_before_sync();
            mbar_arrive(bar_p + half * 8);
        }
    }
    if (ntiles > 0 && act) mbar_wait(bar_done, 0u, err);      // (the others meet these at the next barrier)
    __syncwarp();                                            // warp-aligned barriers and tensor memory follow
    tc_fence_after_sync();

    float bound = 448.f * prun;                              // of |O|
    // What stayed out of the product of the tree's values joins O of the rows that see it, in the stream and the copy that the key's column went to: x 2^(t - R), the score t once
    // more from the rows themselves.  Rare, and small code.
    if (nt > 0 && (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3]) != 0u && (WIDE || half < nt)) {
        unsigned long long odd0 = mk0 & (s_odd[0] | (unsigned long long)s_odd[1] << 32), odd1 = mk1 & (s_odd[2] | (unsigned long long)s_odd[3] << 32);
        if (!WIDE && g0 + half == 0) odd1 = 0ull;
        if (!WIDE && g0 + half == 1) odd0 = 0ull;
        if (REP > 1) {
            const unsigned long long columns = ((1ull << (COLS & 63)) - 1ull) << (copy * COLS & 63);
            odd0 &= columns;
            odd1 &= columns;
        }
        if (__any_sync(HS_FULL_MASK, (odd0 | odd1) != 0ull)) {
#pragma unroll 1
            for (int ch = 0; ch < HS_HEAD_DIM; ch += 16) {
                unsigned int ov[16];
                const unsigned int at = tO + half * HS_HEAD_DIM + lane_off + ch;
                tmem_ld16(at, ov);
                tmem_wait_ld();
#pragma unroll 1
                for (int key = 0; key < nk; ++key) {
                    if (!((key < 64 ? odd0 >> key : odd1 >> (key - 64)) & 1ull)) continue;
                    const size_t kv = ((size_t)kept_row_of(key) * p.c.hkv + h) * HS_HEAD_DIM;
                    float score = 0.f;
#pragma unroll 1
                    for (int c = 0; c < HS_HEAD_DIM; ++c) score = fmaf(__bfloat162float(p.q[(size_t)orow * HS_HEAD_DIM + c]), __bfloat162float(p.k_tree[kv + c]), score);
                    const float weight = fminf(ex2_approx(fmaf(score, p.scale_log2, PG_LIFT - mrun)), 16384.f);      // (huge scores: this one and the product's may differ by more)
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const float x = __bfloat162float(p.v_tree[kv + ch + c]);
                        if (!(fabsf(x) < __uint_as_float(PG_APART))) ov[c] = __float_as_uint(__uint_as_float(ov[c]) + (fabsf(x) < __uint_as_float(PG_ENDLESS) ? weight * x : x * CUDART_INF_F));
                    }
                }
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const float o = fabsf(__uint_as_float(ov[c]));
                    if (o < CUDART_INF_F) bound = fmaxf(bound, o);
                }
                __syncwarp();
                tmem_st16(at, ov);
            }
            tmem_wait_st();
        }
        tc_fence_before_sync();
    }
    // ---- up to 128 rows: the streams and copies of a row are combined like splits -----------------------------------------------------------
    float w0 = 1.f, w1 = 0.f;
    if (!WIDE) {
        float* s_mx = reinterpret_cast<float*>(gen + Y::x);
        float* s_lx = s_mx + 2 * PG_BM;
        float* s_px = reinterpret_cast<float*>(gen + Y::part);       // (the tiles of who has a row are done with)
        s_mx[half * PG_BM + lane_row] = mrun;
        s_lx[half * PG_BM + lane_row] = lrun;
        if (act) s_px[half * PG_BM + lane_row] = bound;
        named_bar_sync(1, PG_SM_THREADS);
        tc_fence_after_sync();
        mrun = -CUDART_INF_F;
#pragma unroll
        for (int k = 0; k < 2 * REP; ++k) mrun = fmaxf(mrun, s_mx[k * (REP > 1 ? ROWS : PG_BM) + row]);
        const float muse = (mrun == -CUDART_INF_F) ? 0.f : mrun;
        w0 = ex2_approx(s_mx[lane_row] - muse);
        w1 = ex2_approx(s_mx[PG_BM + lane_row] - muse);
        lrun = 0.f;
        bound = 0.f;
#pragma unroll
        for (int k = 0; k < 2 * REP; ++k) {
            const int at = k * (REP > 1 ? ROWS : PG_BM) + row;
            const float w = ex2_approx(s_mx[at] - muse);
            lrun = fmaf(s_lx[at], w, lrun);
            bound = fmaf(s_px[at], w, bound);
        }
    }
    // The row's O is sent as f16 times 2^-k, with its largest possible value in [2^14, 2^15): a value keeps its eleven bits down to 2^-28 of that, and loses nothing to other rows, or
    // to what this one weighs with nothing.
    const float kx = (float)max((int)(__float_as_uint(fmaxf(bound, 0.f)) >> 23) - 127 - 14, 0);
    // 16 columns of the row's O; up to 128 rows: of the thread's half of the columns, both streams (a stream without tiles has no O)
    constexpr int CH = WIDE ? 8 : 4;
    const int col_base = WIDE ? 0 : half * 64;
    auto load_o = [&](int ch, float* ov) {
        const unsigned int at = tO + lane_off + col_base + ch * 16;
        unsigned int oa[16], ob[16];
        if (WIDE) {
            if (ntiles > 0) tmem_ld16(at + half * HS_HEAD_DIM, oa);
        } else {
            if (ntiles > 0) tmem_ld16(at, oa);
            if (ntiles > 1) tmem_ld16(at + HS_HEAD_DIM, ob);
        }
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            float v = 0.f;
            if (ntiles > 0) v = WIDE ? __uint_as_float(oa[c]) : __uint_as_float(oa[c]) * w0;
            if (!WIDE && ntiles > 1) v = fmaf(__uint_as_float(ob[c]), w1, v);
            ov[c] = v;
        }
    };
    const float inv = lrun > 0.f ? rcp_approx(lrun) : 0.f;
    // fewer rows than 128: the copies' partials meet in shared memory; items of (row, 8 columns) follow instead of rows
    float* s_part = reinterpret_cast<float*>(gen + Y::part);
    float* s_fin = reinterpret_cast<float*>(gen + Y::x);     // by row: max, sum, 1 / sum, k (over the streams' maxima and sums, which all threads have read)
    if constexpr (REP > 1) {
        named_bar_sync(1, PG_SM_THREADS);
        if (copy == 0 && half == 0) {
            s_fin[row] = mrun;
            s_fin[PG_BM + row] = lrun;
            s_fin[2 * PG_BM + row] = inv;
            s_fin[3 * PG_BM + row] = kx;
        }
#pragma unroll 1
        for (int ch = 0; ch < CH; ++ch) {
            float ov[16];
            load_o(ch, ov);
            if (row < live) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(s_part + lane_row * Y::part_stride + col_base + ch * 16 + q * 4) = make_float4(ov[q * 4], ov[q * 4 + 1], ov[q * 4 + 2], ov[q * 4 + 3]);
            }
            __syncwarp();
        }
        named_bar_sync(1, PG_SM_THREADS);
    }
    auto part8 = [&](int rl, int c8, float* v) {             // 8 columns of row rl, all copies
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
        for (int k = 0; k < REP; ++k) {
            const float4* src = reinterpret_cast<const float4*>(s_part + (k * ROWS + rl) * Y::part_stride + c8 * 8);
            const float4 a = src[0], b4 = src[1];
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b4.x; v[5] += b4.y; v[6] += b4.z; v[7] += b4.w;
        }
    };
    auto out_row = [&](int rl) {
        const int rg = m0 + rl, node = (int)((unsigned int)rg * p.inv_g >> 16);
        return (long long)kept_row_of(node) * p.hq + h * p.G + (rg - node * p.G);
    };

    // ---- epilogue ----------------------------------------------------------------------------------------------------------------------
    if (ns == 1 && REP > 1) {
        for (int it = tid; it < live * 16; it += PG_SM_THREADS) {
            const int rl = it >> 4, c8 = it & 15;
            const float f = s_fin[2 * PG_BM + rl];
            float v[8];
            part8(rl, c8, v);
            const long long og = out_row(rl);
            *reinterpret_cast<uint4*>(p.out + (size_t)og * HS_HEAD_DIM + c8 * 8) =
                make_uint4(pg_pack(v[0] * f, v[1] * f), pg_pack(v[2] * f, v[3] * f), pg_pack(v[4] * f, v[5] * f), pg_pack(v[6] * f, v[7] * f));
            if (c8 == 0 && p.lse_out) p.lse_out[og] = (s_fin[rl] - PG_LIFT + log2f(s_fin[PG_BM + rl])) * LN2;
        }
    } else if (ns == 1) {
#pragma unroll 1
        for (int ch = 0; ch < CH && act; ++ch) {
            float ov[16];
            load_o(ch, ov);
            uint4 o[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                o[q].x = pg_pack(ov[q * 8 + 0] * inv, ov[q * 8 + 1] * inv);
                o[q].y = pg_pack(ov[q * 8 + 2] * inv, ov[q * 8 + 3] * inv);
                o[q].z = pg_pack(ov[q * 8 + 4] * inv, ov[q * 8 + 5] * inv);
                o[q].w = pg_pack(ov[q * 8 + 6] * inv, ov[q * 8 + 7] * inv);
            }
            // two lanes change a chunk each, so that a lane pair writes 32 bytes of a row at a time
            const bool up = (lane & 1) != 0;
            uint4 x = up ? o[0] : o[1];
            x.x = __shfl_xor_sync(HS_FULL_MASK, x.x, 1); x.y = __shfl_xor_sync(HS_FULL_MASK, x.y, 1);
            x.z = __shfl_xor_sync(HS_FULL_MASK, x.z, 1); x.w = __shfl_xor_sync(HS_FULL_MASK, x.w, 1);
            if (up) o[0] = x; else o[1] = x;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int dst = __shfl_sync(HS_FULL_MASK, (int)orow, (lane & ~1) + i);
                if (dst >= 0) *(reinterpret_cast<uint4*>(p.out + (size_t)dst * HS_HEAD_DIM + col_base + ch * 16) + (lane & 1)) = o[i];
            }
        }
        if (orow >= 0 && p.lse_out && (WIDE || half == 0)) p.lse_out[orow] = (mrun - PG_LIFT + log2f(lrun)) * LN2;
    } else {
        // Row rl of the block's live ones is merged by CTA rl * ns / live.  Every thread sends its part of its row, {O 2^-k in f16, max, sum, k}, from registers into the owner's
        // receive area by asynchronous stores that complete on the owner's barrier.  A sender may leave at once.
        const unsigned char* po = gen + Y::recv;
        const unsigned int s_recv = base + Y::recv;
        const int rows_max = (live + ns - 1) / ns + 1;
        if (WIDE) cluster_arrive();                          // every CTA is through with its tiles
        cluster_wait();
        if constexpr (REP > 1) {
            for (int it = tid; it < live * 16; it += PG_SM_THREADS) {
                const int rl = it >> 4, c8 = it & 15;
                const int owner = rl * ns / live, o_lo = (owner * live + ns - 1) / ns;
                const unsigned int dst = cluster_map_addr(s_recv + (unsigned int)(split * rows_max + rl - o_lo) * PG_ROW_STRIDE, owner);
                const unsigned int rbar = cluster_map_addr(bar_r, owner);
                const float k = s_fin[3 * PG_BM + rl], f = power_of_two(-(int)k);
                float v[8];
                part8(rl, c8, v);
                if (c8 == 0) st_async_v4(dst + HS_HEAD_DIM * 2, __float_as_uint(s_fin[rl]), __float_as_uint(s_fin[PG_BM + rl]), __float_as_uint(k), 0u, rbar);
                st_async_v4(dst + c8 * 16, pg_pack_half(v[0] * f, v[1] * f), pg_pack_half(v[2] * f, v[3] * f), pg_pack_half(v[4] * f, v[5] * f), pg_pack_half(v[6] * f, v[7] * f), rbar);
            }
        } else if (act) {
            const int rb = (WIDE ? half * PG_BM : 0) + row;
            const int owner = min(rb, live - 1) * ns / live, o_lo = (owner * live + ns - 1) / ns;
            const bool send = rb < live;
            const unsigned int dst = cluster_map_addr(s_recv + (unsigned int)(split * rows_max + rb - o_lo) * PG_ROW_STRIDE, owner);
            const unsigned int rbar = cluster_map_addr(bar_r, owner);
            if (send && (WIDE || half == 0))
                st_async_v4(dst + HS_HEAD_DIM * 2, __float_as_uint(mrun), __float_as_uint(lrun), __float_as_uint(kx), 0u, rbar);
            const float f = power_of_two(-(int)kx);
#pragma unroll 1
            for (int ch = 0; ch < CH; ++ch) {
                float ov[16];
                load_o(ch, ov);
#pragma unroll
                for (int q = 0; q < 2 && send; ++q)
                    st_async_v4(dst + (col_base + ch * 16 + q * 8) * 2, pg_pack_half(ov[q * 8 + 0] * f, ov[q * 8 + 1] * f), pg_pack_half(ov[q * 8 + 2] * f, ov[q * 8 + 3] * f),
                                pg_pack_half(ov[q * 8 + 4] * f, ov[q * 8 + 5] * f), pg_pack_half(ov[q * 8 + 6] * f, ov[q * 8 + 7] * f), rbar);
            }
        }
        mbar_wait_cluster(bar_r, 0u, err);
        // Half a warp per owned row: a lane weighs the split of its number, then takes eight columns of all of them.
        for (int rl = tid >> 4; rl - (tid >> 4 & 1) < r_hi - r_lo; rl += PG_SM_THREADS / 16) {
            const int s2 = tid & 15;
            const unsigned char* from = po + (size_t)rl * PG_ROW_STRIDE;         // (split 0)
            float4 t = make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
            if (s2 < ns && rl < r_hi - r_lo) t = *reinterpret_cast<const float4*>(from + (size_t)(s2 * rows_max) * PG_ROW_STRIDE + HS_HEAD_DIM * 2);
            float Mx = t.x;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) Mx = fmaxf(Mx, __shfl_xor_sync(HS_FULL_MASK, Mx, o));
            // (a sum that is NaN stays one, also where no score was a number)
            float w = t.x == -CUDART_INF_F && !(t.y != t.y) ? 0.f : ex2_approx(t.x - Mx);
            float lsum = w * t.y;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) lsum += __shfl_xor_sync(HS_FULL_MASK, lsum, o);
            w *= (lsum > 0.f ? rcp_approx(lsum) : lsum) * power_of_two((int)t.z);
            float acc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll 1
            for (int k = 0; k < ns; ++k) {
                const float wk = __shfl_sync(HS_FULL_MASK, w, (lane & 16) + k);
                uint4 v = make_uint4(0, 0, 0, 0);
                if (rl < r_hi - r_lo) v = *reinterpret_cast<const uint4*>(from + (size_t)(k * rows_max) * PG_ROW_STRIDE + s2 * 16);
                const float2 a0 = pg_halves(v.x), a1 = pg_halves(v.y), a2 = pg_halves(v.z), a3 = pg_halves(v.w);
                acc[0] = fmaf(wk, a0.x, acc[0]); acc[1] = fmaf(wk, a0.y, acc[1]); acc[2] = fmaf(wk, a1.x, acc[2]); acc[3] = fmaf(wk, a1.y, acc[3]);
                acc[4] = fmaf(wk, a2.x, acc[4]); acc[5] = fmaf(wk, a2.y, acc[5]); acc[6] = fmaf(wk, a3.x, acc[6]); acc[7] = fmaf(wk, a3.y, acc[7]);
            }
            if (rl < r_hi - r_lo) {
                const long long og = out_row(r_lo + rl);
                *reinterpret_cast<uint4*>(p.out + (size_t)og * HS_HEAD_DIM + s2 * 8) =
                    make_uint4(pg_pack(acc[0], acc[1]), pg_pack(acc[2], acc[3]), pg_pack(acc[4], acc[5]), pg_pack(acc[6], acc[7]));
                if (s2 == 0 && p.lse_out) p.lse_out[og] = (Mx - PG_LIFT + log2f(lsum)) * LN2;
            }
        }
    }
    tc_fence_before_sync();
    named_bar_sync(1, PG_SM_THREADS);
    tc_fence_after_sync();
    if (warp == 0) tmem_dealloc(tmem, PG_TMEM_COLS);
}

// ---- host side -----------------------------------------------------------------------------------------------------
typedef CUresult (*encode_tiled_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                    const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <int ROWS>
static hs_status prepare(const hs_ctx* ctx, int* cap) {
    const auto kernel = tree_attn_paged_kernel<ROWS>;
    cudaFuncAttributes fa;
    // (with fewer registers at launch the softmax warps would wait for theirs for good)
    if (cudaFuncGetAttributes(&fa, kernel) != cudaSuccess || fa.numRegs < PG_REGS) return HS_ERR_CUDA;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<ROWS>::bytes) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
        return HS_ERR_CUDA;
    for (int sz = 1; sz <= PG_MAX_SPLIT; ++sz) {              // CTAs that run at once in clusters of sz
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1, sz, ctx->sm_count);
        cfg.blockDim = dim3(PG_THREADS);
        cfg.dynamicSmemBytes = Layout<ROWS>::bytes;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 1; at[0].val.clusterDim.y = sz; at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) cap[sz] = n * sz;
        else { cap[sz] = 0; (void)cudaGetLastError(); }
    }
    return HS_OK;
}

hs_status hs_launch_attention_paged(hs_ctx* ctx, const hs_pruned_tree* pruned, const hs_kv_cache* cache,
                                    const hs_paged_attn_desc* d, const void* q, const void* k_tree, const void* v_tree,
                                    void* out, float* lse_out, cudaStream_t stream) {
    if (!ctx->paged_ready) {
        for (const auto f : {prepare<32>, prepare<64>, prepare<256>, prepare<128>})
            if (f(ctx, ctx->paged_cap) != HS_OK) return HS_ERR_CUDA;
        ctx->paged_ready = true;
    }
    PagedParams p;
    p.c = kv_pages(cache, ctx->counters + HS_CNT_ERROR);
    p.q = (const __nv_bfloat16*)q;
    p.k_tree = (const __nv_bfloat16*)k_tree;
    p.v_tree = (const __nv_bfloat16*)v_tree;
    p.out = (__nv_bfloat16*)out;
    p.lse_out = lse_out;
    p.n_keep = pruned->n_keep;
    p.keep_off = pruned->keep_off;
    p.keep_idx = pruned->keep_idx;
    p.status = pruned->status;
    p.node_off = d->node_off;
    p.anc_mask = (const unsigned long long*)pruned->anc_mask;
    p.hq = d->hq;
    p.G = d->hq / cache->hkv;
    p.inv_g = (65536u + p.G - 1) / p.G;
    p.layout = d->layout;
    p.max_nodes = d->max_nodes;
    p.max_rows = d->max_rows;
    p.scale_log2 = d->sm_scale * LOG2E;
    const int tiles = (d->max_kv_len + PG_BN - 1) / PG_BN + (d->max_nodes + PG_BN - 1) / PG_BN;
    const PagedChoice how = paged_choice(cache->batch * cache->hkv, p.G * d->max_nodes, ctx->sm_count, tiles, ctx->paged_cap);
    p.nsplit = how.splits;
    const dim3 grid((p.G * d->max_nodes + how.rows - 1) / how.rows, how.splits, cache->batch * cache->hkv);
    // the keys as a matrix of 128-byte rows, a page's rows of one head (or 64 of them) at a time
    CUtensorMap tmK;
    const cuuint64_t gdim[2] = {HS_HEAD_DIM, (cuuint64_t)cache->n_pages * cache->hkv * cache->page_size}, gstr[1] = {HS_HEAD_DIM};
    const cuuint32_t box[2] = {HS_HEAD_DIM, (cuuint32_t)(cache->page_size < PG_BN ? cache->page_size : PG_BN)}, estr[2] = {1, 1};
    if (((encode_tiled_fn)ctx->encode_tiled)(&tmK, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, cache->k, gdim, gstr, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return HS_ERR_CUDA;
    const auto kernel = how.rows == 32 ? tree_attn_paged_kernel<32> : how.rows == 64 ? tree_attn_paged_kernel<64> : how.rows == 128 ? tree_attn_paged_kernel<128>
                        : tree_attn_paged_kernel<256>;
    const cudaError_t e = hs_launch(kernel, grid, dim3(PG_THREADS), how.rows == 256 ? Layout<256>::bytes : Layout<128>::bytes, stream, ctx->pdl,
                                    dim3(1, how.splits, 1), p, tmK);
    return e == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}
