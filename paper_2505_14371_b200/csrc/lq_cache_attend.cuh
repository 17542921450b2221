// Attention of one new token a sequence over the quantised cache: out = sum_j softmax_j(scale q . k_j) v_j.
//
// Mathematics.  A row of the cache is N * level[symbol] with sign.  The keys' norm is a factor of the score and the values'
// norm one of the weight, so the two products run on bare signed levels, which are fp16 numbers as they stand:
//   s_j = (scale N_j) (q . level(K_j)),  w_j = exp2(s_j + log2 M_j - ref'),  out = sum_j w_j level(V_j) / sum_j p_j * 2^(ref' - ref)
// with p_j = exp2(s_j - ref).  Weights and denominator have running references of their own (ref' of s + log2 M, ref of s), so
// that no spread of the values' norms costs a weight its bits; a reference moves only when a score passes it by more than
// kSlack, which the threads of a warp vote on, and sums are rescaled then.  Scores, p, w and all sums are fp32.  Roundings to
// fewer bits: q as fp16 after a power of two per query (exact for fp16 and bf16 queries; rotated and fp32 ones are taken as
// a sum of two fp16 numbers, 22 bits), and w as fp16, 11 bits, for the second product (with fp32 outputs as a sum of two as
// well): the rounding of a weight is at most an eighth of the output's own for bf16 and equal to it for fp16, and independent
// from token to token.
//
// Work.  A warp takes 16 tokens of one head at a time: the keys are the A operand (16 tokens x 16 coordinates) of
// mma.m16n8k16, 8 queries the B operand; the scores' fragment, transposed by two movmatrix, is the B operand of the second
// product, whose A operand is the values transposed (16 coordinates x 16 tokens).  Which coordinate is which column of A is
// free as long as q follows, so lanes read runs of a row as it lies in the page.  tcgen05 would take its operands
// from shared memory or tensor memory, that is the decoded values written out once more; here they go from the look-up
// into the operand's register, and the products are a small part of the time (group <= 8 rows of a 128-row tile).
//
// Decoding.  A byte of a row is looked up in a table of 256 words: two coordinates of 4 bits as one half2 or one of 8 bits.
// The table is in shared memory 32 times, a copy in the bank of each lane, so a look-up has no bank conflict and is
// one byte permute (byte index and lane to address) and one load for two coordinates.  Values need two TOKENS of one
// coordinate in a register: with 4 bits two rows' words are merged into bytes of the two tokens (4 instructions for 16
// coordinates) before the look-up.
//
// Split.  Units of 128 tokens (8 warps x 16) of all (sequence, head, 8 queries) in a row are dealt out evenly to a grid that
// the GPU holds at once; every CTA finds its share from the lengths, on the device.  A CTA that has all of a
// segment (sequence, head, 8 queries) writes its output; the others leave partial sums in the workspace, at most two a CTA, and the CTA
// where a segment begins leaves a record of it, from which a second kernel joins them in the order of the CTAs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lq_cache.cuh"

namespace lq {
namespace attend {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kTile = 16;               // tokens of a warp at a time
constexpr int kQueries = 8;             // queries a segment
constexpr int kTableBytes = 256 * 256;  // entry e: 32 copies for the keys, 32 for the values
constexpr float kLow = -1e30f;          // a reference before its first score
constexpr float kSlack = 8.0f;          // how far (log2) a score may pass its reference
constexpr float kLift = 6.0f;           // weights are 2^kLift at their reference: at most 2^14 as fp16, and exact down to 2^-20

// Workspace: `grid` records of 16 bytes, then 2 * grid partials of kQueries * (padded + 4) floats (sums; reference, reference
// of the weights, denominator, unused).
struct Record { int32_t sequence, head_block, last, pad; };
static_assert(sizeof(Record) == kCacheRecordBytes && kQueries == 8, "the workspace is sized by lq_cache.cuh");
template <int P>
constexpr int64_t kPartial = cache_partial_floats(P);

template <int P>
__host__ __device__ constexpr int combine_bytes() { return kWarps * 2 * 4 * (P + 4) * 4; }
template <int P>
__host__ __device__ constexpr int smem_bytes() { return kTableBytes + combine_bytes<P>() + 2 * kQueries * (P + 8) * 2 + (kQueries + kWarps * kQueries * 3 + kQueries * (kWarps + 4) + 64) * 4; }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float lg2(float x) { float y; asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transposed(uint32_t m)
{
    uint32_t t;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(m));
    return t;
}

__device__ __forceinline__ uint32_t halves(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const uint32_t&>(h);
}

__device__ __forceinline__ float2 rest_of(uint32_t rounded, float lo, float hi)
{
    const float2 r = __half22float2(reinterpret_cast<const __half2&>(rounded));
    return make_float2(lo - r.x, hi - r.y);
}

// The table's word for byte kByte of `w`; lane_base: 4 * lane (+ 128 for the values).
template <int kByte>
__device__ __forceinline__ uint32_t look(const char* table, uint32_t w, uint32_t lane_base)
{
    return *reinterpret_cast<const uint32_t*>(table + __byte_perm(w, lane_base, 0x5504 | (kByte << 4)));
}

__device__ __forceinline__ float load_any(const CacheRows& r, int64_t at)
{
    if (r.type == LQ_F32) return static_cast<const float*>(r.data)[at];
    if (r.type == LQ_F16) return __half2float(static_cast<const __half*>(r.data)[at]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(r.data)[at]);
}

__device__ __forceinline__ void store_any(const CacheRows& r, int64_t at, float v)
{
    if (r.type == LQ_F32) static_cast<float*>(r.data)[at] = v;
    else if (r.type == LQ_F16) static_cast<__half*>(r.data)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(r.data)[at] = __float2bfloat16_rn(v);
}

// What a sequence has to be read of: tokens [first, length), as tiles [tile0, tile1), and units of them.
struct Extent {
    int64_t first, length;
    int64_t tile0, tile1;
    __device__ __forceinline__ int64_t units() const { return (tile1 - tile0 + kWarps - 1) / kWarps; }
};

__device__ __forceinline__ Extent extent_of(const CacheAttendArgs& a, int sequence)
{
    Extent e;
    e.length = __ldg(a.lengths + sequence);
    const int64_t most = a.table_width << a.shape.page_shift;
    if (e.length < 0) e.length = 0;
    if (e.length > most) e.length = most;
    e.first = a.window > 0 && e.length > a.window ? e.length - a.window : 0;
    e.tile0 = e.first / kTile;
    e.tile1 = (e.length + kTile - 1) / kTile;
    return e;
}

// Codes and norms of one tile, as one warp's lanes hold them.
template <int P, int WK, int WV>
struct Tile {
    static constexpr int kKeyBytes = P * WK / 8 / 4, kValueBytes = P * WV / 8 / 8;         // a lane's share of a row
    static constexpr int kKeyChunk = kKeyBytes < 16 ? kKeyBytes : 16, kValueChunk = kValueBytes < 16 ? kValueBytes : 16;
    static constexpr int kKeyChunks = kKeyBytes / kKeyChunk, kValueChunks = kValueBytes / kValueChunk;
    uint32_t k[2][kKeyBytes / 4];       // rows lane / 4 and lane / 4 + 8
    uint32_t v[4][kValueBytes / 4];     // rows 2t, 2t+1, 2t+8, 2t+9 with t = lane % 4
    float nk[2], nv[2];                 // norms of rows lane / 4 and lane / 4 + 8
};

template <int kBytes>
__device__ __forceinline__ void load_run(uint32_t* to, const uint32_t* from)
{
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(to) = __ldg(reinterpret_cast<const uint4*>(from));
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(to) = __ldg(reinterpret_cast<const uint2*>(from));
    else *to = __ldg(from);
}

template <int P, int WK, int WV>
__device__ __forceinline__ void load_tile(Tile<P, WK, WV>& t, const CacheAttendArgs& a, int page, int row0, int head, int lane)
{
    using X = Tile<P, WK, WV>;
    constexpr int kRowK = P * WK / 32, kRowV = P * WV / 32;
    if (page < 0) {                     // not there: the tile's tokens are masked; its codes have to be something
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < X::kKeyBytes / 4; ++i) t.k[r][i] = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < X::kValueBytes / 4; ++i) t.v[r][i] = 0;
        t.nk[0] = t.nk[1] = t.nv[0] = t.nv[1] = 0.0f;
        return;
    }
    const int page_size = 1 << a.shape.page_shift, g = lane >> 2, q = lane & 3;
    const uint32_t* base = a.pages + page * a.shape.page_words + head * a.shape.head_words;
    const uint32_t* keys = base + (row0 + g) * kRowK;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < X::kKeyChunks; ++c)
            load_run<X::kKeyChunk>(&t.k[r][c * X::kKeyChunk / 4], keys + 8 * r * kRowK + (4 * c + q) * (X::kKeyChunk / 4));
    const uint32_t* values = base + page_size * kRowK + (row0 + 2 * q) * kRowV;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < X::kValueChunks; ++c)
            load_run<X::kValueChunk>(&t.v[r][c * X::kValueChunk / 4],
                                     values + ((r & 1) + 8 * (r >> 1)) * kRowV + (8 * c + g) * (X::kValueChunk / 4));
    const float* norms = reinterpret_cast<const float*>(base + page_size * (kRowK + kRowV)) + row0 + g;
    t.nk[0] = __ldg(norms); t.nk[1] = __ldg(norms + 8);
    t.nv[0] = __ldg(norms + page_size); t.nv[1] = __ldg(norms + page_size + 8);
}

// kExact 0: q is one fp16 number; 1: a sum of two; 2: q and the weights are.
template <int P, int WK, int WV, int kExact>
struct Sums {
    float acc[P / 16][4];
    float ref[2], ref_w[2], total[2];   // of queries 2t and 2t + 1
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < P / 16; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
        ref[0] = ref[1] = ref_w[0] = ref_w[1] = kLow;
        total[0] = total[1] = 0.0f;
    }
};

// First product: the 16 x 8 scores of a tile before their factors.
template <int P, int WK, int WV, bool kTwo>
__device__ __forceinline__ void scores(float (&c)[4], const Tile<P, WK, WV>& t, const uint32_t (&q)[P / 16][2],
                                       const uint32_t (&q2)[kTwo ? P / 16 : 1][2], const char* table, uint32_t lane_base)
{
    c[0] = c[1] = c[2] = c[3] = 0.0f;
#pragma unroll
    for (int s = 0; s < P / 16; ++s) {
        uint32_t a0, a1, a2, a3;
        if constexpr (WK == 4) {
            const uint32_t w0 = t.k[0][s / 2], w1 = t.k[1][s / 2];
            if (s % 2 == 0) {
                a0 = look<0>(table, w0, lane_base); a2 = look<1>(table, w0, lane_base);
                a1 = look<0>(table, w1, lane_base); a3 = look<1>(table, w1, lane_base);
            } else {
                a0 = look<2>(table, w0, lane_base); a2 = look<3>(table, w0, lane_base);
                a1 = look<2>(table, w1, lane_base); a3 = look<3>(table, w1, lane_base);
            }
        } else {
            const uint32_t w0 = t.k[0][s], w1 = t.k[1][s];
            a0 = __byte_perm(look<0>(table, w0, lane_base), look<1>(table, w0, lane_base), 0x5410);
            a2 = __byte_perm(look<2>(table, w0, lane_base), look<3>(table, w0, lane_base), 0x5410);
            a1 = __byte_perm(look<0>(table, w1, lane_base), look<1>(table, w1, lane_base), 0x5410);
            a3 = __byte_perm(look<2>(table, w1, lane_base), look<3>(table, w1, lane_base), 0x5410);
        }
        mma(c, a0, a1, a2, a3, q[s][0], q[s][1]);
        if constexpr (kTwo) mma(c, a0, a1, a2, a3, q2[s][0], q2[s][1]);
    }
}

// Second product: acc[m] += values^T x weights.  Lane (g, t) has coordinates of row g of A: even ones, of row g + 8: odd ones.
template <int P, int WK, int WV, bool kTwo>
__device__ __forceinline__ void weigh(float (&acc)[P / 16][4], const Tile<P, WK, WV>& t, const uint32_t (&b)[2],
                                      const uint32_t (&b2)[2], const char* table, uint32_t lane_base)
{
    auto step = [&](int m, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
        mma(acc[m], a0, a1, a2, a3, b[0], b[1]);
        if constexpr (kTwo) mma(acc[m], a0, a1, a2, a3, b2[0], b2[1]);
    };
#pragma unroll
    for (int i = 0; i < Tile<P, WK, WV>::kValueBytes / 4; ++i) {
        const uint32_t w0 = t.v[0][i], w1 = t.v[1][i], w2 = t.v[2][i], w3 = t.v[3][i];
        if constexpr (WV == 4) {
            const uint32_t e = (w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), o = ((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u);
            const uint32_t e2 = (w2 & 0x0f0f0f0fu) | ((w3 << 4) & 0xf0f0f0f0u), o2 = ((w2 >> 4) & 0x0f0f0f0fu) | (w3 & 0xf0f0f0f0u);
            step(4 * i, look<0>(table, e, lane_base), look<0>(table, o, lane_base), look<0>(table, e2, lane_base), look<0>(table, o2, lane_base));
            step(4 * i + 1, look<1>(table, e, lane_base), look<1>(table, o, lane_base), look<1>(table, e2, lane_base), look<1>(table, o2, lane_base));
            step(4 * i + 2, look<2>(table, e, lane_base), look<2>(table, o, lane_base), look<2>(table, e2, lane_base), look<2>(table, o2, lane_base));
            step(4 * i + 3, look<3>(table, e, lane_base), look<3>(table, o, lane_base), look<3>(table, e2, lane_base), look<3>(table, o2, lane_base));
        } else {
            auto two = [&](uint32_t x, uint32_t y) { return __byte_perm(x, y, 0x5410); };
            step(2 * i, two(look<0>(table, w0, lane_base), look<0>(table, w1, lane_base)), two(look<1>(table, w0, lane_base), look<1>(table, w1, lane_base)),
                 two(look<0>(table, w2, lane_base), look<0>(table, w3, lane_base)), two(look<1>(table, w2, lane_base), look<1>(table, w3, lane_base)));
            step(2 * i + 1, two(look<2>(table, w0, lane_base), look<2>(table, w1, lane_base)), two(look<3>(table, w0, lane_base), look<3>(table, w1, lane_base)),
                 two(look<2>(table, w2, lane_base), look<2>(table, w3, lane_base)), two(look<3>(table, w2, lane_base), look<3>(table, w3, lane_base)));
        }
    }
}

// Coordinate of A's row g (row g + 8: the next one) in tile m of the second product.
template <int P, int WV>
__device__ __forceinline__ int value_coordinate(int m, int g)
{
    constexpr int kBytes = P * WV / 8 / 8, kChunk = kBytes < 16 ? kBytes : 16, kEach = kChunk * 8 / WV;   // coordinates a chunk
    const int c = 2 * m / kEach;
    return (8 * c + g) * kEach + 2 * m % kEach;
}

// First coordinate of the four that lane t gives to step s of the first product.
template <int P, int WK>
__device__ __forceinline__ int key_coordinate(int s, int t)
{
    constexpr int kBytes = P * WK / 8 / 4, kChunk = kBytes < 16 ? kBytes : 16, kEach = kChunk * 8 / WK;
    const int c = 4 * s / kEach;
    return (4 * c + t) * kEach + 4 * s % kEach;
}

// Where the shared memory's parts are.
template <int P>
struct Shared {
    char* table;
    float* combine;                     // [warp][query % 2][query / 2][P + 4]
    __half* q;                          // [2][kQueries][P + 8]: q, and what its rounding left
    float* factor;                      // [kQueries]: scale * log2(e) / the query's power of two
    float* stats;                       // [warp][kQueries][3]
    float* share;                       // [kQueries][kWarps + 4]: factor of each warp's sums; then ref, ref_w, total
    int64_t* words;                     // [32] for the schedule
    __device__ explicit Shared(char* s)
    {
        table = s;
        combine = reinterpret_cast<float*>(s + kTableBytes);
        words = reinterpret_cast<int64_t*>(s + kTableBytes + combine_bytes<P>());
        q = reinterpret_cast<__half*>(words + 32);
        factor = reinterpret_cast<float*>(q + 2 * kQueries * (P + 8));
        stats = factor + kQueries;
        share = stats + kWarps * kQueries * 3;
    }
};

// Warp `w` brings query w of the block into shared memory: rotated, times its power of two, as fp16 and the rest.
template <int P>
__device__ __forceinline__ void stage_query(const Shared<P>& sh, const CacheAttendArgs& a, int sequence, int head, int block, int w, int lane, int64_t length)
{
    const int query = block * kQueries + w;
    float x[P / 32];
    uint32_t top = 0;
    bool lost = false;
    if (query < a.group) {
        const int64_t row = sequence * a.queries.token_stride + (int64_t)(head * a.group + query) * a.queries.head_stride;
        const CacheRotary& r = a.rotary;
        const int half = r.dim / 2;
        const float* cs = r.table;
        if (r.table) {
            const int64_t at = r.at ? __ldg(r.at + sequence) : (length > 0 ? length - 1 : 0);
            lost = at < 0 || at >= r.positions;
            if (!lost) cs += at * r.dim;
        }
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            const int d = lane + 32 * i;
            x[i] = d < a.shape.dim ? load_any(a.queries, row + d) : 0.0f;
            if (r.table && d < r.dim && !lost) {
                const bool first = r.interleaved ? d % 2 == 0 : d < half;
                const int other = r.interleaved ? d ^ 1 : first ? d + half : d - half;
                const int p = r.interleaved ? d / 2 : first ? d : d - half;
                const float c = __ldg(cs + p), s = __ldg(cs + half + p), y = load_any(a.queries, row + other);
                x[i] = first ? __fsub_rn(__fmul_rn(x[i], c), __fmul_rn(y, s)) : __fadd_rn(__fmul_rn(x[i], c), __fmul_rn(y, s));
            }
            if (lost) x[i] = __uint_as_float(0x7fffffffu);
            top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        }
        if (lost && lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION);
    } else {
#pragma unroll
        for (int i = 0; i < P / 32; ++i) x[i] = 0.0f;
    }
    top = __reduce_max_sync(0xffffffffu, top);
    // 2^e brings the largest coordinate to [2^14, 2^15); Inf and NaN stay what they are
    int e = top >= 0x7f800000u || top == 0 ? 0 : 141 - (int)(top >> 23);
    e = min(e, 120);
    const float up = __uint_as_float((uint32_t)(127 + e) << 23), down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < P / 32; ++i) {
        const float y = x[i] * up;
        const __half h = __float2half_rn(y);
        sh.q[w * (P + 8) + lane + 32 * i] = h;
        sh.q[(kQueries + w) * (P + 8) + lane + 32 * i] = __float2half_rn(y - __half2float(h));
    }
    if (lane == 0) sh.factor[w] = a.scale * down;
}

template <int P, int WK, int WV, int kExact>
__global__ void __launch_bounds__(kThreads, cache_attend_resident(P, WK, WV)) attend_kernel(const __grid_constant__ CacheAttendArgs a)
{
    extern __shared__ __align__(128) char smem[];
    const Shared<P> sh(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

    {   // the look-up table: thread e writes the copies of entry e, a warp's lanes at different banks
        const uint32_t k = __ldg(a.tables[LQ_KEYS].pairs + tid), v = __ldg(a.tables[LQ_VALUES].pairs + tid);
        uint4* row = reinterpret_cast<uint4*>(sh.table + tid * 256);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            row[(j + lane) & 7] = make_uint4(k, k, k, k);
            row[8 + ((j + lane) & 7)] = make_uint4(v, v, v, v);
        }
    }

    // ---- this CTA's share of all units
    const int head_blocks = a.shape.heads * a.group_blocks;
    int64_t sum = 0;
    for (int b = tid; b < a.batch; b += kThreads) {
        sum += extent_of(a, b).units();
        const int n = __ldg(a.lengths + b);
        if (blockIdx.x == 0 && (n < 0 || n > a.table_width << a.shape.page_shift)) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh.words[warp] = sum;
    if (tid == 0) sh.words[16] = -1;
    __syncthreads();
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all += sh.words[w];
    all *= head_blocks;
    // no more CTAs than units take part, so that none between two that share a segment is without a unit
    const int64_t grid = min(all, (int64_t)gridDim.x);
    const int64_t begin = blockIdx.x < grid ? all * blockIdx.x / grid : 0, end = blockIdx.x < grid ? all * (blockIdx.x + 1) / grid : 0;
    Record* records = reinterpret_cast<Record*>(a.partial);
    float* partials = a.partial + (int64_t)gridDim.x * (sizeof(Record) / 4);
    if (tid == 0) records[blockIdx.x].sequence = -1;

    if (begin < end) {
        // the sequence that unit `begin` belongs to, and the units before it
        int64_t before = 0;
        for (int base = 0; base < a.batch; base += kThreads) {
            const int b = base + tid;
            const int64_t mine = b < a.batch ? extent_of(a, b).units() * head_blocks : 0;
            int64_t scan = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t up = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += up;
            }
            __syncthreads();
            if (lane == 31) sh.words[warp] = scan;
            __syncthreads();
            int64_t whole = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                if (w == warp) scan += before + whole;
                whole += sh.words[w];
            }
            if (begin >= scan - mine && begin < scan) { sh.words[16] = b; sh.words[17] = scan - mine; }
            before += whole;
            if (before > begin) break;
        }
        __syncthreads();
        int sequence = (int)sh.words[16];
        Extent x = extent_of(a, sequence);
        int64_t units = x.units();
        const int64_t offset = begin - sh.words[17];
        int hb = (int)(offset / units);
        int64_t chunk = offset - hb * units, at = begin;
        const uint32_t base_k = 4 * lane, base_v = 128 + 4 * lane;
        const int tile_shift = a.shape.page_shift - 4;

        while (at < end) {
            const int64_t count = min(units - chunk, end - at);        // units of this segment that are ours
            const int head = hb / a.group_blocks, block = hb - head * a.group_blocks;
            __syncthreads();                                            // the last segment's shared memory has been read
            stage_query<P>(sh, a, sequence, head, block, warp, lane, x.length);
            __syncthreads();
            uint32_t q[P / 16][2], q2[kExact ? P / 16 : 1][2];
#pragma unroll
            for (int s = 0; s < P / 16; ++s) {
                const uint2 w = *reinterpret_cast<const uint2*>(sh.q + g * (P + 8) + key_coordinate<P, WK>(s, t));
                q[s][0] = w.x; q[s][1] = w.y;
                if constexpr (kExact > 0) {
                    const uint2 w2 = *reinterpret_cast<const uint2*>(sh.q + (kQueries + g) * (P + 8) + key_coordinate<P, WK>(s, t));
                    q2[s][0] = w2.x; q2[s][1] = w2.y;
                }
            }
            const float f0 = sh.factor[2 * t], f1 = sh.factor[2 * t + 1];

            Sums<P, WK, WV, kExact> S;
            S.clear();
            const int32_t* row = a.table + (int64_t)sequence * a.table_width;
            auto page_of = [&](int64_t tile) {
                const int p = __ldg(row + (tile >> tile_shift));
                if (p >= 0 && p < a.num_pages) return p;
                if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_PAGE);
                return -1;
            };
            int64_t tile = x.tile0 + chunk * kWarps + warp;
            const int64_t stop = min(x.tile1, x.tile0 + (chunk + count) * kWarps);
            Tile<P, WK, WV> cur, next;
            int page = -1, page_next = -1, page_after = -1;
            if (tile < stop) { page = page_of(tile); }
            if (tile + kWarps < stop) page_next = page_of(tile + kWarps);
            if (tile < stop) load_tile<P, WK, WV>(cur, a, page, (int)(tile & ((1 << tile_shift) - 1)) * kTile, head, lane);
            for (; tile < stop; tile += kWarps) {
                const bool more = tile + kWarps < stop;
                if (tile + 2 * kWarps < stop) page_after = page_of(tile + 2 * kWarps);
                if (more) load_tile<P, WK, WV>(next, a, page_next, (int)((tile + kWarps) & ((1 << tile_shift) - 1)) * kTile, head, lane);

                float c[4];
                scores<P, WK, WV, (kExact > 0)>(c, cur, q, q2, sh.table, base_k);
                const int64_t token = tile * kTile + g;
                const bool in0 = page >= 0 && token >= x.first && token < x.length;
                const bool in1 = page >= 0 && token + 8 >= x.first && token + 8 < x.length;
                const float s0 = in0 ? c[0] * (f0 * cur.nk[0]) : -INFINITY, s1 = in0 ? c[1] * (f1 * cur.nk[0]) : -INFINITY;
                const float s2 = in1 ? c[2] * (f0 * cur.nk[1]) : -INFINITY, s3 = in1 ? c[3] * (f1 * cur.nk[1]) : -INFINITY;
                const float lv0 = in0 ? lg2(cur.nv[0]) : -INFINITY, lv1 = in1 ? lg2(cur.nv[1]) : -INFINITY;
                const float w0 = s0 + lv0, w1 = s1 + lv0, w2 = s2 + lv1, w3 = s3 + lv1;
                const float top0 = fmaxf(s0, s2), top1 = fmaxf(s1, s3), topw0 = fmaxf(w0, w2), topw1 = fmaxf(w1, w3);
                const bool passed = top0 > S.ref[0] + kSlack || top1 > S.ref[1] + kSlack || topw0 > S.ref_w[0] + kSlack || topw1 > S.ref_w[1] + kSlack;
                if (__any_sync(0xffffffffu, passed)) {
                    float m[4] = {top0, top1, topw0, topw1};
#pragma unroll
                    for (int o = 4; o < 32; o *= 2)
#pragma unroll
                        for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float r = fmaxf(S.ref[i], m[i]), rw = fmaxf(S.ref_w[i], m[2 + i]);
                        S.total[i] *= ex2(S.ref[i] - r);
                        const float f = ex2(S.ref_w[i] - rw);
                        S.ref[i] = r; S.ref_w[i] = rw;
#pragma unroll
                        for (int k = 0; k < P / 16; ++k) { S.acc[k][i] *= f; S.acc[k][2 + i] *= f; }
                    }
                }
                S.total[0] += ex2(s0 - S.ref[0]) + ex2(s2 - S.ref[0]);
                S.total[1] += ex2(s1 - S.ref[1]) + ex2(s3 - S.ref[1]);
                const float e0 = ex2(w0 - S.ref_w[0] + kLift), e1 = ex2(w1 - S.ref_w[1] + kLift);
                const float e2 = ex2(w2 - S.ref_w[0] + kLift), e3 = ex2(w3 - S.ref_w[1] + kLift);
                const uint32_t h0 = halves(e0, e1), h1 = halves(e2, e3);
                const uint32_t b[2] = {transposed(h0), transposed(h1)};
                uint32_t b2[2] = {0, 0};
                if constexpr (kExact == 2) {
                    const float2 r0 = rest_of(h0, e0, e1), r1 = rest_of(h1, e2, e3);
                    b2[0] = transposed(halves(r0.x, r0.y));
                    b2[1] = transposed(halves(r1.x, r1.y));
                }
                weigh<P, WK, WV, (kExact == 2)>(S.acc, cur, b, b2, sh.table, base_v);
                if (more) cur = next;
                page = page_next; page_next = page_after;
            }

            // ---- the warps' sums added up
#pragma unroll
            for (int o = 4; o < 32; o *= 2) {
                S.total[0] += __shfl_xor_sync(0xffffffffu, S.total[0], o);
                S.total[1] += __shfl_xor_sync(0xffffffffu, S.total[1], o);
            }
            if (g == 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float* st = sh.stats + (warp * kQueries + 2 * t + i) * 3;
                    st[0] = S.ref[i]; st[1] = S.ref_w[i]; st[2] = S.total[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float* to = sh.combine + ((warp * 2 + i) * 4 + t) * (P + 4);
#pragma unroll
                for (int m = 0; m < P / 16; m += 2)
                    *reinterpret_cast<float4*>(to + value_coordinate<P, WV>(m, g)) =
                        make_float4(S.acc[m][i], S.acc[m][2 + i], S.acc[m + 1][i], S.acc[m + 1][2 + i]);
            }
            __syncthreads();
            if (tid < kQueries) {
                float r = kLow, rw = kLow, total = 0.0f;
                for (int w = 0; w < kWarps; ++w) {
                    const float* st = sh.stats + (w * kQueries + tid) * 3;
                    r = fmaxf(r, st[0]); rw = fmaxf(rw, st[1]);
                }
                for (int w = 0; w < kWarps; ++w) {
                    const float* st = sh.stats + (w * kQueries + tid) * 3;
                    total += st[2] * ex2(st[0] - r);
                    sh.share[tid * (kWarps + 4) + w] = ex2(st[1] - rw);
                }
                float* o = sh.share + tid * (kWarps + 4) + kWarps;
                o[0] = r; o[1] = rw; o[2] = total;
            }
            __syncthreads();
            const bool starts = chunk == 0, whole = starts && chunk + count == units;
            const int slot = 2 * blockIdx.x + starts;
            for (int i = tid; i < kQueries * P / 4; i += kThreads) {
                const int query = i / (P / 4), d = (i % (P / 4)) * 4;
                const float* share = sh.share + query * (kWarps + 4);
                float4 sum4 = make_float4(0, 0, 0, 0);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(sh.combine + ((w * 2 + (query & 1)) * 4 + (query >> 1)) * (P + 4) + d);
                    const float f = share[w];
                    sum4.x += v.x * f; sum4.y += v.y * f; sum4.z += v.z * f; sum4.w += v.w * f;
                }
                const float r = share[kWarps], rw = share[kWarps + 1], total = share[kWarps + 2];
                if (whole) {
                    if (block * kQueries + query < a.group) {
                        const float f = total != 0.0f ? ex2(rw - r - kLift) / total : 0.0f;
                        const int64_t to = sequence * a.out.token_stride + (int64_t)(head * a.group + block * kQueries + query) * a.out.head_stride;
                        const float o[4] = {sum4.x * f, sum4.y * f, sum4.z * f, sum4.w * f};
#pragma unroll
                        for (int k = 0; k < 4; ++k) if (d + k < a.shape.dim) store_any(a.out, to + d + k, o[k]);
                        if (d == 0 && a.lse)
                            a.lse[(int64_t)sequence * a.shape.heads * a.group + head * a.group + block * kQueries + query] =
                                total != 0.0f ? (r + log2f(total)) * 0.693147180559945309f : -INFINITY;
                    }
                } else {
                    float* to = partials + slot * kPartial<P> + query * (P + 4);
                    *reinterpret_cast<float4*>(to + d) = sum4;
                    if (d == 0) *reinterpret_cast<float4*>(to + P) = make_float4(r, rw, total, 0.0f);
                }
            }
            if (starts && !whole && tid == 0) {
                // the CTA that has the segment's last unit: the largest c whose share begins at or before it
                const int64_t unit = at + units - 1;
                const int64_t c = ((unit + 1) * grid - 1) / all;
                Record rec;
                rec.sequence = sequence; rec.head_block = hb; rec.last = (int32_t)c; rec.pad = 0;
                records[blockIdx.x] = rec;
            }
            at += count;
            chunk = 0;
            if (at < end && ++hb == head_blocks) {
                hb = 0;
                do { x = extent_of(a, ++sequence); units = x.units(); } while (units == 0);
            }
        }
    }

    // sequences without a token to see
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (extent_of(a, b).units() > 0) continue;
        const int queries = a.shape.heads * a.group;
        for (int64_t i = tid; i < (int64_t)queries * a.shape.dim; i += kThreads)
            store_any(a.out, b * a.out.token_stride + (i / a.shape.dim) * a.out.head_stride + i % a.shape.dim, 0.0f);
        if (a.lse) for (int i = tid; i < queries; i += kThreads) a.lse[(int64_t)b * queries + i] = -INFINITY;
    }
}

// Joins the partial sums of a segment that began in CTA `blockIdx.x` and went on in others; a warp a query.
template <int P>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(const __grid_constant__ CacheAttendArgs a)
{
    const Record rec = reinterpret_cast<const Record*>(a.partial)[blockIdx.x];
    if (rec.sequence < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = rec.head_block / a.group_blocks, query = (rec.head_block - head * a.group_blocks) * kQueries + warp;
    if (query >= a.group) return;
    const float* partials = a.partial + (int64_t)gridDim.x * (sizeof(Record) / 4) + warp * (P + 4);
    auto part = [&](int c) { return partials + (2 * (int64_t)c + (c == (int)blockIdx.x)) * kPartial<P>; };
    float r = kLow, rw = kLow;
    for (int c = blockIdx.x + lane; c <= rec.last; c += 32) {
        const float4 st = *reinterpret_cast<const float4*>(part(c) + P);
        r = fmaxf(r, st.x); rw = fmaxf(rw, st.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        r = fmaxf(r, __shfl_xor_sync(0xffffffffu, r, o));
        rw = fmaxf(rw, __shfl_xor_sync(0xffffffffu, rw, o));
    }
    float total = 0.0f, acc[P / 32] = {};
#pragma unroll 4
    for (int c = blockIdx.x; c <= rec.last; ++c) {
        const float* p = part(c);
        const float4 st = *reinterpret_cast<const float4*>(p + P);
        total += st.z * ex2(st.x - r);
        const float f = ex2(st.y - rw);
#pragma unroll
        for (int i = 0; i < P / 32; ++i) acc[i] += p[lane + 32 * i] * f;
    }
    const float f = total != 0.0f ? ex2(rw - r - kLift) / total : 0.0f;
    const int64_t to = rec.sequence * a.out.token_stride + (int64_t)(head * a.group + query) * a.out.head_stride;
#pragma unroll
    for (int i = 0; i < P / 32; ++i) if (lane + 32 * i < a.shape.dim) store_any(a.out, to + lane + 32 * i, acc[i] * f);
    if (lane == 0 && a.lse)
        a.lse[(int64_t)rec.sequence * a.shape.heads * a.group + head * a.group + query] =
            total != 0.0f ? (r + log2f(total)) * 0.693147180559945309f : -INFINITY;
}

template <int P, int WK, int WV, int kExact>
cudaError_t launch_as(const CacheAttendArgs& a, cudaStream_t s)
{
    const cudaError_t e = cudaFuncSetAttribute(attend_kernel<P, WK, WV, kExact>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<P>());
    if (e != cudaSuccess) return e;
    attend_kernel<P, WK, WV, kExact><<<a.grid, kThreads, smem_bytes<P>(), s>>>(a);
    if (a.split) attend_join_kernel<P><<<a.grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

template <int P, int WK, int WV>
cudaError_t launch_exact(const CacheAttendArgs& a, cudaStream_t s)
{
    if (a.queries.type == LQ_F32) return launch_as<P, WK, WV, 2>(a, s);
    return a.rotary.table ? launch_as<P, WK, WV, 1>(a, s) : launch_as<P, WK, WV, 0>(a, s);
}

template <int P>
cudaError_t launch(const CacheAttendArgs& a, cudaStream_t s)
{
    if (a.shape.sym_bits[0] == 4) return a.shape.sym_bits[1] == 4 ? launch_exact<P, 4, 4>(a, s) : launch_exact<P, 4, 8>(a, s);
    return a.shape.sym_bits[1] == 4 ? launch_exact<P, 8, 4>(a, s) : launch_exact<P, 8, 8>(a, s);
}

}  // namespace attend
}  // namespace lq
