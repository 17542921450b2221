// Attention of one new token a sequence over the quantised cache: out = sum_j softmax_j(scale q . k_j) v_j.
//
// Mathematics.  A row of the cache is N * level[symbol] with sign.  The keys' norm is a factor of the score and the values'
// norm one of the weight, so the two products run on bare signed levels, which are fp16 numbers as they stand:
//   s_j = (scale N_j) (q . level(K_j)),  w_j = exp2((s_j - ref) + (log2 M_j - k)),  out = 2^k sum_j w_j level(V_j) / sum_j p_j
// with p_j = exp2(s_j - ref).  Weights have a scale 2^k beside the running reference of the scores, so that no spread of the values'
// norms costs a weight its bits; k is a whole number and s_j - ref is formed first, so that neither large scores nor large logarithms
// round the sum.  Reference and scale move only when an exponent passes kSlack, which the threads of a warp vote on, and sums are
// rescaled then.  Scores, p, w and all sums are fp32.  Roundings to fewer bits: q as fp16 after a power of two per query (exact for
// fp16 and bf16 queries; rotated and fp32 ones are taken as a sum of two fp16 numbers, 22 bits), and w, for the second product of bf16
// outputs as fp16, 11 bits (at most an eighth of the output's own rounding, and independent from token to token), of fp16 and fp32
// ones as a sum of two, 22 bits (of a weight down to 2^-9 of the largest; below, to 2^-31 of the largest).
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
// Feeding.  The codes and norms of a tile are four runs of a page.  A warp copies them by 16-byte cp.async into stages of shared
// memory of its own, kStages tiles deep, so nothing but a wait for its own copies stands between warps.  In a stage the tokens are four
// groups of 4 rows with a gap behind each, and the tile's tokens are dealt to the rows of the operands (token_row) such that
// both the keys' and the values' reads meet every bank once.
//
// Split.  Units of 128 tokens (8 warps x 16; 256 where a warp takes two tiles at a time) of all (sequence, head, 8 queries) in a
// row are dealt out evenly to teams of 8 warps, as many as the GPU holds at once (two a CTA, which share the look-up table;
// one for rows of 256); every team finds its share from the lengths, on the device.  The start of a segment (sequence, head,
// 8 queries) counts as two units more: 64 sequences of 250 to 16384 tokens 110 -> 89 us.  A team that has all of a segment writes its
// output; the others leave partial sums in the workspace, at most two a team, and the team where a segment begins leaves a
// record of it, from which a second kernel joins them in the order of the teams, so that the same call gives the same bits.
//
// Loads.  Both kernels start beside their predecessor, which may be what writes the lengths, pages, queries or partial sums: what is
// read behind pdl_wait is read by ordinary loads, by cp.async, or by intrinsics on a pointer from fresh().
//
// What bounds it: shared memory, which a tile of 16 tokens and 128 coordinates of 4 bits keeps busy for 108 cycles (88 of loads, 64 of
// them look-ups, and 20 of copies and sums written), where DRAM would need 93; 63 % of its cycles are used, and 62 % of the issue slots, as
// the 16 warps of an SM wait for their own results.  64 sequences of 250 to 16384 tokens, 8 heads of 128 in 4 bits: 89 us, where the copy
// bandwidth would take 45.6.  Short sequences: a segment's chain of page, copy, products, sum and output, some 4 us.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

namespace lq {
namespace attend {

constexpr int kTeamWarps = 8;
constexpr int kTeam = 32 * kTeamWarps;  // threads
constexpr int kTile = 16;               // tokens of a warp at a time
constexpr int kQueries = 8;             // queries a segment
constexpr int kTableBytes = 256 * 256;  // entry e: 32 copies for the keys, 32 for the values
// Shared memory, by address: 64 KB below the table hold stages of some warps, the table starts at 64 KB, so that a byte of a row
// is the second byte of its entry's address, behind it come the other warps' stages.  (The first KB of a CTA's shared memory is the
// system's; the last one that a CTA can have is left free, so that the places below hold wherever in the first the kernel's own begins.)
constexpr int kTableAt = 1 << 16, kSystemBytes = 1 << 10, kEnd = (227 << 10);
constexpr int kStart = 2;               // what a segment costs beside its units, in units
constexpr float kLow = -3.402823466e38f;    // the reference of a warp or team without a score: below every finite score's
constexpr float kSlack = 8.0f;          // how far (log2) a score may pass its reference, a weight its scale
constexpr float kLift = 6.0f;           // weights are 2^kLift at their scale: at most 2^14 as fp16 (2^15 times a significand), with all bits down to 2^-20 of it
template <bool kFloat>
constexpr float kLiftOf = kFloat ? 0.0f : kLift;    // ... of it in the exponent (otherwise in the significand)

// Workspace: a record for every team, then two partials of kCacheRecordBytes a team (sums; reference, scale of the weights,
// denominator, unused).
struct Record { int32_t sequence, head_block, last, pad; };
static_assert(sizeof(Record) == kCacheRecordBytes && kQueries == 8, "the workspace is sized by lq_cache.cuh");
template <int P>
constexpr int64_t kPartial = cache_partial_floats(P);

template <int P>
struct TeamShared {
    int64_t words[18];                  // schedule
    float factor[kQueries];             // scale * log2(e) / the query's power of two
    float stats[kTeamWarps][kQueries][3];
    float share[kQueries][kTeamWarps + 4];      // factor of each warp's sums; then that of the whole segment's
    alignas(16) __half q[2][kQueries][P + 8];   // the queries, and what their rounding left
};
template <int P>
constexpr int kTeamSharedBytes = (int)sizeof(TeamShared<P>);

// A tile of one warp in shared memory: keys, values, 16 norms of keys, 16 of values.
template <int P, int WK, int WV>
struct Stage {
    static constexpr int kRowK = P * WK / 8, kRowV = P * WV / 8;                            // bytes
    // Gap behind each group of 4 rows.  Values: lane t's rows sit in group t or t ^ 1, and a phase of a read takes 32 bytes
    // of each of four rows: 32.  Keys: a phase takes 32 or 64 bytes of rows whose groups are neighbours.
    static constexpr int kGapK = kRowK == 64 ? 0 : 64, kGapV = 32;
    static constexpr int kGroupK = 4 * kRowK + kGapK, kGroupV = 4 * kRowV + kGapV;
    static constexpr int kValues = 4 * kGroupK, kNorms = kValues + 4 * kGroupV, kBytes = kNorms + 8 * kTile;
    static constexpr int kTeams = cache_attend_teams(P), kWarps = kTeams * kTeamWarps;
    static constexpr int kPair = cache_attend_pair(P, WK, WV), kUnit = cache_attend_unit(P, WK, WV);
    // as many stages as fit for all warps, on both sides of the table; behind them a KB for what a team shares
    static constexpr int low(int stages) { return (kTableAt - kSystemBytes) / (stages * kBytes); }
    static constexpr int high(int stages) { return (kEnd - kTableAt - kTableBytes - kTeams * kTeamSharedBytes<P>) / (stages * kBytes); }
    static constexpr int fit() { int n = 6; while (low(n) + high(n) < kWarps) n -= kPair; return n; }
    static constexpr int kStages = fit();
    static constexpr int kWarpBytes = kStages * kBytes, kLow = low(kStages) < kWarps ? low(kStages) : kWarps;
    static constexpr int kTeamsAt = kTableAt + kTableBytes + (kWarps - kLow) * kWarpBytes;
    // Shared address of a warp's stages.
    static __device__ __forceinline__ int stages_at(int warp)
    {
        return warp < kLow ? kSystemBytes + warp * kWarpBytes : kTableAt + kTableBytes + (warp - kLow) * kWarpBytes;
    }
    static constexpr int kSumBytes = kQueries * (P + 4) * 4;                                // a warp's sums, in its stages' place
    static_assert(kStages >= 2 * kPair && kStages % kPair == 0 && kWarpBytes >= kSumBytes && kBytes % 16 == 0, "stages");
};

template <int P, int WK, int WV>
constexpr int smem_bytes() { return Stage<P, WK, WV>::kTeamsAt + Stage<P, WK, WV>::kTeams * kTeamSharedBytes<P>; }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float lg2(float x) { float y; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// The values' norm of a token, 2^x m: for fp32 outputs its exponent and significand (with 2^kLift), so that a weight is as exact for
// norms of 1e-12 as for 1 (the logarithm's error grows with its size: 6e-6 at 1e12); for others x = log2 and m is not used.
// What is not a positive normal number becomes its logarithm in both: 0 a weight of 0, NaN NaN.
template <bool kFloat>
__device__ __forceinline__ void norm_parts(float norm, float& x, float& m)
{
    x = lg2(norm);
    if constexpr (kFloat) {
        const uint32_t bits = __float_as_uint(norm);
        const float exponent = __uint_as_float(0x4b000000u | bits >> 23) - (8388608.0f + 127.0f);
        if (bits - 0x00800000u < 0x7f000000u) x = exponent;
        m = __uint_as_float((bits & 0x007fffffu) | (127u + (uint32_t)kLift) << 23);
    }
}

// A scale as a whole number, so that its differences from exponents are exact; rounded down, so that the largest weight is 2^kLift or more.
// (The bound takes the place of -infinity; what is that far below the largest p adds nothing to an fp32 output.)
__device__ __forceinline__ float whole_scale(float v) { return floorf(fmaxf(v, -1000.0f)); }

// What the sum of weighted values is multiplied by in the end: 2^scale / total, the power in two factors that are normal numbers.
template <bool kFloat>
__device__ __forceinline__ float out_factor(float scale, float total)
{
    const int n = max((int)scale - (kFloat ? (int)kLift : 0), -252), half = n >> 1;
    const float f = 1.0f / total * __uint_as_float((uint32_t)(127 + half) << 23) * __uint_as_float((uint32_t)(127 + n - half) << 23);
    return total != 0.0f ? f : 0.0f;
}

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

// The table's word for byte kByte of `w`; lane_base: kTableAt + 4 * lane (+ 128 for the values).
template <int kByte>
__device__ __forceinline__ uint32_t look(uint32_t w, uint32_t lane_base)
{
    uint32_t v;                         // (the table does not change once it is there: no need to keep the order of these loads)
    asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(__byte_perm(w, lane_base, 0x7604 | (kByte << 4))));
    return v;
}

__device__ __forceinline__ void copy16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" :: "n"(kLeft) : "memory"); }

// Barrier of one team.
__device__ __forceinline__ void team_sync(int team) { asm volatile("bar.sync %0, %1;" :: "r"(team + 1), "n"(kTeam) : "memory"); }

__device__ __forceinline__ char* row_of(const CacheRows& r, int token, int head)
{
    return static_cast<char*>(r.data) + (int64_t)token * r.token_bytes + (int64_t)head * r.head_bytes;
}

__device__ __forceinline__ void store_any(int type, char* row, int d, float v)
{
    if (type == LQ_F32) reinterpret_cast<float*>(row)[d] = v;
    else if (type == LQ_F16) reinterpret_cast<__half*>(row)[d] = __float2half_rn(v);
    else reinterpret_cast<__nv_bfloat16*>(row)[d] = __float2bfloat16_rn(v);
}

// Coordinates d .. d+3 of an output row.
template <bool kFloat>
__device__ __forceinline__ void store_four(const CacheRows& r, char* row, int d, int dim, float4 v)
{
    if (r.wide && d + 4 <= dim) {
        if constexpr (kFloat) {
            *reinterpret_cast<float4*>(row + 4 * d) = v;
        } else {
            uint2 w;
            if (r.type == LQ_BF16) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
                w = make_uint2(reinterpret_cast<const uint32_t&>(a), reinterpret_cast<const uint32_t&>(b));
            } else {
                w = make_uint2(halves(v.x, v.y), halves(v.z, v.w));
            }
            *reinterpret_cast<uint2*>(row + 2 * d) = w;
        }
        return;
    }
    const float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) if (d + k < dim) store_any(r.type, row, d + k, o[k]);
}

// What a sequence has to be read of: tokens [first, length), as tiles [tile0, tile1).
struct Extent {
    uint32_t first, length;             // (a tile's last token may be just past 2^31)
    int32_t tile0, tile1;
    template <int kUnit>
    __device__ __forceinline__ int64_t units() const { return (tile1 - tile0 + kUnit - 1) / kUnit; }
};

__device__ __forceinline__ Extent extent_of(const CacheAttendArgs& a, int sequence)
{
    Extent e;
    const int64_t most = a.table_width << a.shape.page_shift;
    const int n = a.lengths[sequence];
    e.length = n < 0 ? 0 : n > most ? (uint32_t)most : (uint32_t)n;
    e.first = a.window > 0 && e.length > a.window ? e.length - (uint32_t)a.window : 0;
    e.tile0 = (int32_t)(e.first / kTile);
    e.tile1 = (int32_t)((e.length + kTile - 1) / kTile);
    return e;
}

// Which token of a tile is row r of the operands (row r + 8: two tokens on): rows 2t and 2t + 1, which lane t holds of the
// values, are in groups t and t ^ 1.
__device__ __forceinline__ int token_row(int r)
{
    const int t = r >> 1;
    return (r & 1) ? 4 * (t ^ 1) + 1 : 4 * t;
}

// Copies of tiles into stages.  A lane's pieces of 16 bytes lie at the same places of every tile, so that per tile there is
// little to work out: a tile's keys and values are one run each, and lane i takes the pieces i, i + 32, ...
template <int P, int WK, int WV>
struct Copier {
    using X = Stage<P, WK, WV>;
    const char* codes;                  // the layer's pages, at this lane's first piece
    const char* norms;                  // ... at its piece of the norms (lanes 0 to 3: of the keys', 4 to 7: of the values')
    uint32_t page_bytes, values_at;
    uint32_t to, to_norms;              // shared addresses
    __device__ __forceinline__ Copier(const CacheAttendArgs& a, uint32_t stage0, int lane)
    {
        const char* pages = reinterpret_cast<const char*>(a.pages);
        codes = pages + lane * 16;
        norms = pages + ((X::kRowK + X::kRowV) << a.shape.page_shift) + ((lane & 4) << a.shape.page_shift) + (lane & 3) * 16;
        page_bytes = (uint32_t)a.shape.page_words * 4;
        values_at = X::kRowK << a.shape.page_shift;
        to = stage0;
        to_norms = stage0 + X::kNorms + lane * 16;
    }
    // `head_at`: bytes of a page before the head's part; `lane` as at the start
    __device__ __forceinline__ void tile(int stage, uint32_t page, uint32_t head_at, uint32_t row0, int lane) const
    {
        const int at = stage * X::kBytes;
        const uint64_t from = (uint64_t)page * page_bytes + head_at;
        const char* keys = codes + from + row0 * X::kRowK;
        const char* values = codes + from + values_at + row0 * X::kRowV;
#pragma unroll
        for (int i = 0; i < X::kRowK; i += 32)      // (16 rows are kRow pieces; a group of 4 rows is kRow / 4 of them)
            copy16(to + at + (i + lane) * 16 + (i + lane) / (X::kRowK / 4) * X::kGapK, keys + i * 16);
#pragma unroll
        for (int i = 0; i < X::kRowV; i += 32)
            copy16(to + at + X::kValues + (i + lane) * 16 + (i + lane) / (X::kRowV / 4) * X::kGapV, values + i * 16);
        if (lane < 8) copy16(to_norms + at, norms + from + row0 * 4);
    }
};

// Codes and norms of one tile, as one warp's lanes hold them.
template <int P, int WK, int WV>
struct Tile {
    static constexpr int kKeyBytes = P * WK / 8 / 4, kValueBytes = P * WV / 8 / 8;         // a lane's share of a row
    static constexpr int kKeyChunk = kKeyBytes < 16 ? kKeyBytes : 16, kValueChunk = kValueBytes < 16 ? kValueBytes : 16;
    static constexpr int kKeyChunks = kKeyBytes / kKeyChunk, kValueChunks = kValueBytes / kValueChunk;
    uint32_t k[2][kKeyBytes / 4];       // rows lane / 4 and lane / 4 + 8
    uint32_t v[4][kValueBytes / 4];     // rows 2t, 2t+1, 2t+8, 2t+9 with t = lane % 4
};

template <int kBytes>
__device__ __forceinline__ void take_run(uint32_t* to, const char* from)
{
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(from);
    else *to = *reinterpret_cast<const uint32_t*>(from);
}

// `keys`: the stage, at this lane's place in the row of token_row(lane / 4).
template <int P, int WK, int WV>
__device__ __forceinline__ void take_keys(Tile<P, WK, WV>& t, const char* keys)
{
    using X = Tile<P, WK, WV>;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < X::kKeyChunks; ++c)
            take_run<X::kKeyChunk>(&t.k[r][c * X::kKeyChunk / 4], keys + 2 * r * Stage<P, WK, WV>::kRowK + 4 * c * X::kKeyChunk);
}

// `even`, `odd`: likewise in the rows of token_row(2t) and token_row(2t + 1).
template <int P, int WK, int WV>
__device__ __forceinline__ void take_values(Tile<P, WK, WV>& t, const char* even, const char* odd)
{
    using X = Tile<P, WK, WV>;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < X::kValueChunks; ++c)
            take_run<X::kValueChunk>(&t.v[r][c * X::kValueChunk / 4],
                                     (r & 1 ? odd : even) + (r >> 1) * 2 * Stage<P, WK, WV>::kRowV + 8 * c * X::kValueChunk);
}

// How queries and weights are rounded to fp16.  kPlain: a query is one number (exactly, for fp16 and bf16 that are not rotated), a
// weight one of 11 bits.  kTwo: a query is a sum of two, with a second product for the rest; kWeights: a weight is; kTwoBoth,
// kTwoBothHalf: both are.  With up to 4 queries a head the rests take columns 4 to 7 of the same product (kBeside: of queries,
// kBesideBoth, kBesideHalf: of queries and weights), which costs neither registers nor products: 32 sequences of 8192 tokens, rows of
// 128 in 4 bits, 4 queries a head: rotated bf16 87 -> 77 us, fp16 82 -> 77, fp32 93 -> 81.  (Both: rows of 32 bits, half: of 16.)
// One number is a weight of bf16 outputs: its rounding adds 1 % to the error of the output's own, and two cost 1 to 10 % of the time
// (rows of 128 in 4 bits, 8 queries a head: 75.9 us, 83.8 with two).  With fp16 outputs it would add 39 %.
constexpr int kPlain = 0, kTwo = 1, kTwoBoth = 2, kBeside = 3, kBesideBoth = 4, kBesideHalf = 5, kWeights = 6, kTwoBothHalf = 7;

template <int P>
struct Sums {
    float acc[P / 16][4];
    float ref[2], scale[2], total[2];   // of queries 2t and 2t + 1; the scale is a whole number
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < P / 16; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
        ref[0] = ref[1] = scale[0] = scale[1] = total[0] = total[1] = 0.0f;
    }
};

// First product: the 16 x 8 scores of a tile before their factors.
template <int P, int WK, int WV, bool kTwo>
__device__ __forceinline__ void scores(float (&c)[4], const Tile<P, WK, WV>& t, const uint32_t (&q)[P / 16][2],
                                       const uint32_t (&q2)[kTwo ? P / 16 : 1][2], uint32_t lane_base)
{
    float c2[4] = {};
    c[0] = c[1] = c[2] = c[3] = 0.0f;
#pragma unroll
    for (int s = 0; s < P / 16; ++s) {
        uint32_t a0, a1, a2, a3;
        if constexpr (WK == 4) {
            const uint32_t w0 = t.k[0][s / 2], w1 = t.k[1][s / 2];
            if (s % 2 == 0) {
                a0 = look<0>(w0, lane_base); a2 = look<1>(w0, lane_base);
                a1 = look<0>(w1, lane_base); a3 = look<1>(w1, lane_base);
            } else {
                a0 = look<2>(w0, lane_base); a2 = look<3>(w0, lane_base);
                a1 = look<2>(w1, lane_base); a3 = look<3>(w1, lane_base);
            }
        } else {
            const uint32_t w0 = t.k[0][s], w1 = t.k[1][s];
            a0 = __byte_perm(look<0>(w0, lane_base), look<1>(w0, lane_base), 0x5410);
            a2 = __byte_perm(look<2>(w0, lane_base), look<3>(w0, lane_base), 0x5410);
            a1 = __byte_perm(look<0>(w1, lane_base), look<1>(w1, lane_base), 0x5410);
            a3 = __byte_perm(look<2>(w1, lane_base), look<3>(w1, lane_base), 0x5410);
        }
        mma(c, a0, a1, a2, a3, q[s][0], q[s][1]);
        if constexpr (kTwo) mma(c2, a0, a1, a2, a3, q2[s][0], q2[s][1]);
    }
    if constexpr (kTwo) { c[0] += c2[0]; c[1] += c2[1]; c[2] += c2[2]; c[3] += c2[3]; }
}

// Second product: acc[m] += values^T x weights.  Lane (g, t) has coordinates of row g of A: even ones, of row g + 8: odd ones.
template <int P, int WK, int WV, bool kTwo>
__device__ __forceinline__ void weigh(float (&acc)[P / 16][4], const Tile<P, WK, WV>& t, const uint32_t (&b)[2],
                                      const uint32_t (&b2)[2], uint32_t lane_base)
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
            step(4 * i, look<0>(e, lane_base), look<0>(o, lane_base), look<0>(e2, lane_base), look<0>(o2, lane_base));
            step(4 * i + 1, look<1>(e, lane_base), look<1>(o, lane_base), look<1>(e2, lane_base), look<1>(o2, lane_base));
            step(4 * i + 2, look<2>(e, lane_base), look<2>(o, lane_base), look<2>(e2, lane_base), look<2>(o2, lane_base));
            step(4 * i + 3, look<3>(e, lane_base), look<3>(o, lane_base), look<3>(e2, lane_base), look<3>(o2, lane_base));
        } else {
            auto two = [&](uint32_t x, uint32_t y) { return __byte_perm(x, y, 0x5410); };
            step(2 * i, two(look<0>(w0, lane_base), look<0>(w1, lane_base)), two(look<1>(w0, lane_base), look<1>(w1, lane_base)),
                 two(look<0>(w2, lane_base), look<0>(w3, lane_base)), two(look<1>(w2, lane_base), look<1>(w3, lane_base)));
            step(2 * i + 1, two(look<2>(w0, lane_base), look<2>(w1, lane_base)), two(look<3>(w0, lane_base), look<3>(w1, lane_base)),
                 two(look<2>(w2, lane_base), look<2>(w3, lane_base)), two(look<3>(w2, lane_base), look<3>(w3, lane_base)));
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

// Query w of the block by warp w, in two steps: what has to be fetched is asked for, without a look at it, before the segment's first
// copies, and made into numbers and rotated behind them (in one step the copies came 2000 cycles later).
template <int P, bool kFloat>
struct Query {
    uint32_t x[P / 32], y[P / 32];      // coordinates lane, lane + 32, ... as they are stored, and the partners of rotated ones
    float c[P / 32], s[P / 32];
    bool lost = false;                  // the position is not in the table

    static __device__ __forceinline__ uint32_t raw(const char* row, int d)
    {
        if constexpr (kFloat) return reinterpret_cast<const uint32_t*>(row)[d];
        else return reinterpret_cast<const unsigned short*>(row)[d];
    }
    static __device__ __forceinline__ float number(uint32_t v, int type)
    {
        if constexpr (kFloat) return __uint_as_float(v);
        else return type == LQ_BF16 ? __uint_as_float(v << 16) : __half2float(__ushort_as_half((unsigned short)v));
    }
    __device__ __forceinline__ void fetch(const CacheAttendArgs& a, int sequence, int head, int query, int lane, uint32_t length)
    {
        const CacheRotary& r = a.rotary;
        const bool live = query < a.group;
        const char* const row = row_of(a.queries, sequence, head * a.group + query);
        const float* angles = r.table;
        const int half = r.dim / 2;
        if (r.table && live) {
            const int64_t at = r.at ? r.at[sequence] : (length > 0 ? (int64_t)length - 1 : 0);
            lost = at < 0 || at >= r.positions;
            if (lost) { if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION); }
            else angles += at * r.dim;
        }
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            const int d = lane + 32 * i;
            x[i] = live && d < a.shape.dim ? raw(row, d) : 0;
            y[i] = 0; c[i] = s[i] = 0.0f;       // (a place without a query holds zeros: its scores vote with the others')
            if (r.table && live && !lost && d < r.dim) {
                const int p = r.interleaved ? d / 2 : d < half ? d : d - half;
                c[i] = angles[p]; s[i] = angles[half + p];
                y[i] = raw(row, r.interleaved ? d ^ 1 : d < half ? d + half : d - half);
            }
        }
    }
    __device__ __forceinline__ void finish(float (&out)[P / 32], const CacheAttendArgs& a, int lane) const
    {
        const CacheRotary& r = a.rotary;
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            const int d = lane + 32 * i;
            const float v = number(x[i], a.queries.type);
            out[i] = v;
            if (r.table && d < r.dim) {
                const float u = number(y[i], a.queries.type);
                out[i] = (r.interleaved ? d % 2 == 0 : d < r.dim / 2) ? __fsub_rn(__fmul_rn(v, c[i]), __fmul_rn(u, s[i]))
                                                                     : __fadd_rn(__fmul_rn(v, c[i]), __fmul_rn(u, s[i]));
            }
            if (lost) out[i] = __uint_as_float(0x7fffffffu);
        }
    }
};

// ... and brought into shared memory: times its power of two, as fp16 and the rest; kRests: warps 4 to 7 bring the rests of queries 0 to 3.
template <int P, bool kRests>
__device__ __forceinline__ void stage_query(TeamShared<P>& sh, const float (&x)[P / 32], float scale, int w, int lane)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < P / 32; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    // 2^e brings the largest coordinate to [2^14, 2^15); Inf and NaN stay what they are
    int e = top >= 0x7f800000u || top == 0 ? 0 : 141 - (int)(top >> 23);
    e = min(e, 120);
    const float up = __uint_as_float((uint32_t)(127 + e) << 23), down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < P / 32; ++i) {
        const float y = x[i] * up;
        const __half h = __float2half_rn(y), rest = __float2half_rn(y - __half2float(h));
        sh.q[0][w][lane + 32 * i] = kRests && w >= 4 ? rest : h;
        sh.q[1][w][lane + 32 * i] = rest;
    }
    if (lane == 0) sh.factor[w] = scale * down;
}

template <int P, int WK, int WV, int kMode>
__global__ void __launch_bounds__(Stage<P, WK, WV>::kTeams* kTeam, 1) attend_kernel(const __grid_constant__ CacheAttendArgs a)
{
    using X = Stage<P, WK, WV>;
    using T = Tile<P, WK, WV>;
    constexpr bool kSecond = kMode == kTwo || kMode == kTwoBoth || kMode == kTwoBothHalf, kRestsBoth = kMode == kBesideBoth || kMode == kBesideHalf;
    constexpr bool kRests = kMode == kBeside || kRestsBoth, kWeighTwo = kMode == kTwoBoth || kMode == kTwoBothHalf || kMode == kWeights;
    constexpr bool kFloat = kMode == kTwoBoth || kMode == kBesideBoth;
    extern __shared__ __align__(128) char smem[];
    char* const shared = smem - __cvta_generic_to_shared(smem);         // shared address 0
    char* const table = shared + kTableAt;
    const int team = threadIdx.x / kTeam, tid = threadIdx.x % kTeam, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    char* const stages = shared + X::stages_at(team * kTeamWarps + warp);
    TeamShared<P>& sh = reinterpret_cast<TeamShared<P>*>(shared + X::kTeamsAt)[team];

    {   // the look-up table: a thread writes copies of one entry, a warp's lanes at different banks
        const bool mine = X::kTeams == 1 || team == 0, other = X::kTeams == 1 || team == 1;
        const uint32_t k = mine ? a.tables[LQ_KEYS].pairs[tid] : 0, v = other ? a.tables[LQ_VALUES].pairs[tid] : 0;
        uint4* row = reinterpret_cast<uint4*>(table + tid * 256);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (mine) row[(j + lane) & 7] = make_uint4(k, k, k, k);
            if (other) row[8 + ((j + lane) & 7)] = make_uint4(v, v, v, v);
        }
    }
    pdl_wait();
    pdl_launch_next();

    // ---- this team's share of all units
    const int head_blocks = a.shape.heads * a.group_blocks, me = blockIdx.x * X::kTeams + team, teams = gridDim.x * X::kTeams;
    // what the segments of sequence `b` cost: units, and kStart for each segment that has any
    auto units_of = [&](int b) -> int64_t {
        const int64_t u = b < a.batch ? extent_of(a, b).template units<X::kUnit>() : 0;
        return u ? (u + kStart) * head_blocks : 0;
    };
    auto warp_scan = [&](int64_t v) {
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t up = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += up;
        }
        return v;
    };
    // the first kTeam sequences, which are all of most batches, are scanned once; the rest only counted here
    const int64_t mine0 = units_of(tid);
    int64_t scan0 = warp_scan(mine0), rest = 0;
    for (int b = tid + kTeam; b < a.batch; b += kTeam) rest += units_of(b);
    if (a.batch > kTeam) rest = warp_scan(rest);
    if (lane == 31) { sh.words[warp] = scan0; sh.words[kTeamWarps + warp] = rest; }
    if (me == 0)
        for (int b = tid; b < a.batch; b += kTeam) {
            const int n = a.lengths[b];
            if (n < 0 || n > a.table_width << a.shape.page_shift) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
        }
    __syncthreads();                    // (the table is there too)
    int64_t all = 0, before = 0;        // units of all sequences, and of the first kTeam
#pragma unroll
    for (int w = 0; w < kTeamWarps; ++w) {
        if (w == warp) scan0 += before;
        before += sh.words[w];
        all += sh.words[kTeamWarps + w];
    }
    all += before;
    // no more teams than units take part, so that none between two that share a segment is without a unit
    const int64_t parts = min(all, (int64_t)teams);
    auto share_of = [&](int i) -> int64_t {     // (a division of 64 bits takes some 200 cycles)
        return all < 1 << 20 ? (int64_t)((uint32_t)all * (uint32_t)i / (uint32_t)parts) : all * i / parts;
    };
    const int64_t begin = me < parts ? share_of(me) : 0, end = me < parts ? share_of(me + 1) : 0;
    Record* records = reinterpret_cast<Record*>(a.partial);
    float* partials = a.partial + (int64_t)teams * (sizeof(Record) / 4);
    if (tid == 0 && a.partial) records[me].sequence = -1;

    if (begin < end) {
        // the sequence that unit `begin` belongs to, and the units before it
        auto found = [&](int b, int64_t mine, int64_t scan) {
            if (begin >= scan - mine && begin < scan) { sh.words[16] = b; sh.words[17] = scan - mine; }
        };
        found(tid, mine0, scan0);
        for (int base = kTeam; before <= begin; base += kTeam) {
            const int64_t mine = units_of(base + tid);
            int64_t scan = warp_scan(mine);
            team_sync(team);
            if (lane == 31) sh.words[warp] = scan;
            team_sync(team);
#pragma unroll
            for (int w = 0; w < kTeamWarps; ++w) {
                if (w == warp) scan += before;
                before += sh.words[w];
            }
            found(base + tid, mine, scan);
        }
        team_sync(team);
        int sequence = (int)sh.words[16];
        Extent extent = extent_of(a, sequence);
        int64_t units = extent.template units<X::kUnit>();
        const int64_t offset = begin - sh.words[17];
        int hb = offset < 1 << 30 ? (int)((uint32_t)offset / (uint32_t)(units + kStart)) : (int)(offset / (units + kStart));
        int64_t chunk = offset - hb * (units + kStart) - kStart, at = begin;      // below 0: what comes before the segment's first unit

        const uint32_t base_k = kTableAt + 4 * lane, base_v = base_k + 128, stage0 = (uint32_t)X::stages_at(team * kTeamWarps + warp);
        const Copier<P, WK, WV> copier(a, stage0, lane);
        const int tile_shift = a.shape.page_shift - 4, tile_mask = (1 << tile_shift) - 1;
        // this lane's places in a stage
        const int row = token_row(g), row_even = token_row(2 * t), row_odd = token_row(2 * t + 1);
        const char* const keys = stages + (row >> 2) * X::kGroupK + (row & 3) * X::kRowK + t * T::kKeyChunk;
        const char* const even = stages + X::kValues + (row_even >> 2) * X::kGroupV + (row_even & 3) * X::kRowV + g * T::kValueChunk;
        const char* const odd = stages + X::kValues + (row_odd >> 2) * X::kGroupV + (row_odd & 3) * X::kRowV + g * T::kValueChunk;
        const char* const norms = stages + X::kNorms + row * 4;

        while (at < end) {
            const int64_t ours = min(units - chunk, end - at);
            const int count = (int)(ours + min(chunk, (int64_t)0));     // units of this segment that are ours
            if (count <= 0) break;                                      // (the end of our share)
            if (chunk < 0) chunk = 0;
            const int head = hb / a.group_blocks, block = hb - head * a.group_blocks;
            // ---- the first copies: this warp's tiles are kPair of every unit
            const int32_t* pages = a.table + (int64_t)sequence * a.table_width;
            const int tile0 = extent.tile0 + (int)chunk * X::kUnit + warp * X::kPair, stop = min(extent.tile1, extent.tile0 + ((int)chunk + count) * X::kUnit);
            const int rounds = stop > tile0 ? (stop - tile0 + X::kUnit - 1) / X::kUnit : 0;
            const uint32_t head_at = (uint32_t)(head * a.shape.head_words) * 4;
            auto tile_of = [&](int n) { return tile0 + n / X::kPair * X::kUnit + n % X::kPair; };      // of the warp's n-th tile
            uint32_t missing = 0;                                       // bit s: stage s holds no tile: past the end, or on a page that is not there
            int page = -1;                                              // lane l: of the warp's tile 32 i + l, i as far as copies are
            auto page_of = [&](int n) { const int tile = tile_of(n); return tile < stop ? pages[tile >> tile_shift] : -1; };
            const int first_pages = page_of(lane);
            Query<P, kFloat> query_raw;
            query_raw.fetch(a, sequence, head, block * kQueries + (kRests ? warp % 4 : warp), lane, extent.length);
            auto start = [&](int round, int stage) {
                if (round < rounds) {
                    if (round * X::kPair % 32 == 0) {
                        page = round == 0 ? first_pages : page_of(round * X::kPair + lane);
                        if (page < 0 || page >= a.num_pages) {
                            if (tile_of(round * X::kPair + lane) < stop) atomicOr(a.flags, LQ_CACHE_BAD_PAGE);
                            page = -1;
                        }
                    }
#pragma unroll
                    for (int h = 0; h < X::kPair; ++h) {
                        const int n = round * X::kPair + h, p = __shfl_sync(0xffffffffu, page, n % 32);
                        missing = p < 0 ? missing | 1u << (stage + h) : missing & ~(1u << (stage + h));
                        if (p >= 0) copier.tile(stage + h, (uint32_t)p, head_at, (uint32_t)(tile_of(n) & tile_mask) * kTile, lane);
                    }
                }
                commit_copies();
            };
            for (int j = 0; j < X::kStages / X::kPair - 1; ++j) start(j, j * X::kPair);
            float mine[P / 32];
            query_raw.finish(mine, a, lane);
            stage_query<P, kRests>(sh, mine, a.scale, warp, lane);
            team_sync(team);
            uint32_t q[P / 16][2], q2[kSecond ? P / 16 : 1][2];
#pragma unroll
            for (int s = 0; s < P / 16; ++s) {
                const uint2 w = *reinterpret_cast<const uint2*>(&sh.q[0][g][key_coordinate<P, WK>(s, t)]);
                q[s][0] = w.x; q[s][1] = w.y;
                if constexpr (kSecond) {
                    const uint2 w2 = *reinterpret_cast<const uint2*>(&sh.q[1][g][key_coordinate<P, WK>(s, t)]);
                    q2[s][0] = w2.x; q2[s][1] = w2.y;
                }
            }
            const float f0 = sh.factor[2 * t], f1 = sh.factor[2 * t + 1];

            Sums<P> S;
            S.clear();
            bool begun = false;                                         // the reference is a score's
            int stage = 0, ahead = X::kStages - X::kPair;
            for (int j = 0; j < rounds; ++j) {
                __syncwarp();                                           // every lane has read the stages that are filled next
                start(j + X::kStages / X::kPair - 1, ahead);
                wait_copies<X::kStages / X::kPair - 1>();
                __syncwarp();
                const int place = stage * X::kBytes;
                const uint32_t gone = missing >> stage & ((1u << X::kPair) - 1);
                if ((stage += X::kPair) == X::kStages) stage = 0;
                if ((ahead += X::kPair) == X::kStages) ahead = 0;
                if (gone == (1u << X::kPair) - 1) continue;

                // exponents of p and of the weights; the values' norms as 2^x m
                float d[X::kPair][4], w[X::kPair][4], m[X::kPair][2];
#pragma unroll
                for (int h = 0; h < X::kPair; ++h) {
                    T cur;
                    float c[4];
                    take_keys(cur, keys + place + h * X::kBytes);
                    scores<P, WK, WV, kSecond>(c, cur, q, q2, base_k);
                    if constexpr (kRests)               // columns 4 to 7 are the rests of columns 0 to 3
#pragma unroll
                        for (int i = 0; i < 4; ++i) c[i] += __shfl_xor_sync(0xffffffffu, c[i], 2);
                    const char* n = norms + place + h * X::kBytes;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float nk = *reinterpret_cast<const float*>(n + 8 * r);
                        float x;
                        norm_parts<kFloat>(*reinterpret_cast<const float*>(n + 64 + 8 * r), x, m[h][r]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            d[h][2 * r + i] = fmaf(c[2 * r + i] * (i ? f1 : f0), nk, -S.ref[i]);
                            w[h][2 * r + i] = d[h][2 * r + i] + (x - S.scale[i]);
                        }
                    }
                }
                const uint32_t first = (uint32_t)(tile0 + j * X::kUnit) * kTile;
                if (gone || first < extent.first || first + X::kPair * kTile > extent.length) {     // the ends of what is seen
#pragma unroll
                    for (int h = 0; h < X::kPair; ++h)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const uint32_t token = first + h * kTile + row + i;
                            if ((gone >> h & 1) || token < extent.first || token >= extent.length) d[h][i] = d[h][i + 1] = w[h][i] = w[h][i + 1] = -INFINITY;
                        }
                }
                T values;                       // the first tile's before what the scores go through (1 to 2 % where there are two)
                take_values(values, even + place, odd + place);
                float top_d = -INFINITY, top_w = -INFINITY;
#pragma unroll
                for (int h = 0; h < X::kPair; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) { top_d = fmaxf(top_d, d[h][i]); top_w = fmaxf(top_w, w[h][i]); }
                if (__any_sync(0xffffffffu, top_d > kSlack || top_w > kSlack + kLiftOf<kFloat> || !begun)) {
                    float x[X::kPair][2];
#pragma unroll
                    for (int h = 0; h < X::kPair; ++h)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {   // (once more, so that they need not be kept)
                            float unused;
                            norm_parts<kFloat>(*reinterpret_cast<const volatile float*>(norms + place + h * X::kBytes + 64 + 8 * r), x[h][r], unused);
                        }
                    float step[2], moved[2], scale[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        step[i] = begun ? 0.0f : -INFINITY; scale[i] = -INFINITY;
#pragma unroll
                        for (int h = 0; h < X::kPair; ++h) step[i] = fmaxf(step[i], fmaxf(d[h][i], d[h][2 + i]));
                    }
                    auto over_tokens = [](float (&v)[2]) {              // the largest of the lanes with the same queries
#pragma unroll
                        for (int o = 4; o < 32; o *= 2)
#pragma unroll
                            for (int i = 0; i < 2; ++i) v[i] = fmaxf(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
                    };
                    over_tokens(step);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float ref = step[i] > -INFINITY ? S.ref[i] + step[i] : S.ref[i];
                        moved[i] = S.ref[i] - ref;
                        S.ref[i] = ref;
#pragma unroll
                        for (int h = 0; h < X::kPair; ++h)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                d[h][2 * r + i] += moved[i];
                                scale[i] = fmaxf(scale[i], d[h][2 * r + i] == -INFINITY ? -INFINITY : d[h][2 * r + i] + x[h][r]);
                            }
                    }
                    over_tokens(scale);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float k = whole_scale(begun ? fmaxf(S.scale[i] + moved[i], scale[i] - kLiftOf<kFloat>) : scale[i] - kLiftOf<kFloat>);
#pragma unroll
                        for (int h = 0; h < X::kPair; ++h)
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                w[h][2 * r + i] = d[h][2 * r + i] == -INFINITY ? -INFINITY : d[h][2 * r + i] + (x[h][r] - k);
                        if (begun) {
                            S.total[i] *= ex2(moved[i]);
                            const float f = ex2(moved[i] + (S.scale[i] - k));
#pragma unroll
                            for (int m = 0; m < P / 16; ++m) { S.acc[m][i] *= f; S.acc[m][2 + i] *= f; }
                        }
                        S.scale[i] = k;
                    }
                    begun = true;
                }
#pragma unroll
                for (int h = 0; h < X::kPair; ++h) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        S.total[i & 1] += ex2(d[h][i]);
                        w[h][i] = ex2(w[h][i]);
                        if constexpr (kFloat) w[h][i] *= m[h][i >> 1];
                    }
                    uint32_t h0 = halves(w[h][0], w[h][1]), h1 = halves(w[h][2], w[h][3]);
                    if constexpr (kRestsBoth) {
                        const float2 r0 = rest_of(h0, w[h][0], w[h][1]), r1 = rest_of(h1, w[h][2], w[h][3]);
                        if (t >= 2) { h0 = halves(r0.x, r0.y); h1 = halves(r1.x, r1.y); }
                    }
                    const uint32_t b[2] = {transposed(h0), transposed(h1)};
                    uint32_t b2[2] = {0, 0};
                    if constexpr (kWeighTwo) {
                        const float2 r0 = rest_of(h0, w[h][0], w[h][1]), r1 = rest_of(h1, w[h][2], w[h][3]);
                        b2[0] = transposed(halves(r0.x, r0.y));
                        b2[1] = transposed(halves(r1.x, r1.y));
                    }
                    if (h > 0) take_values(values, even + place + h * X::kBytes, odd + place + h * X::kBytes);
                    weigh<P, WK, WV, kWeighTwo>(S.acc, values, b, b2, base_v);
                }
            }

            // ---- the warps' sums added up, through the stages
#pragma unroll
            for (int o = 4; o < 32; o *= 2) {
                S.total[0] += __shfl_xor_sync(0xffffffffu, S.total[0], o);
                S.total[1] += __shfl_xor_sync(0xffffffffu, S.total[1], o);
            }
            if (g == 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float* st = sh.stats[warp][2 * t + i];
                    st[0] = begun ? S.ref[i] : kLow; st[1] = S.scale[i]; st[2] = S.total[i];
                }
            }
            wait_copies<0>();
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float* to = reinterpret_cast<float*>(stages) + (i * 4 + t) * (P + 4);
#pragma unroll
                for (int m = 0; m < P / 16; m += 2)
                    *reinterpret_cast<float4*>(to + value_coordinate<P, WV>(m, g)) =
                        make_float4(S.acc[m][i], S.acc[m][2 + i], S.acc[m + 1][i], S.acc[m + 1][2 + i]);
            }
            team_sync(team);
            const bool starts = chunk == 0, whole = starts && count == units;
            const int slot = 2 * me + starts;
            if (tid < kQueries) {
                float r = kLow, scale = -INFINITY, total = 0.0f;
                for (int w = 0; w < kTeamWarps; ++w) r = fmaxf(r, sh.stats[w][tid][0]);
                for (int w = 0; w < kTeamWarps; ++w) scale = fmaxf(scale, sh.stats[w][tid][1] + (sh.stats[w][tid][0] - r));
                scale = whole_scale(scale);
                for (int w = 0; w < kTeamWarps; ++w) {
                    const float moved = sh.stats[w][tid][0] - r;
                    total += sh.stats[w][tid][2] * ex2(moved);
                    sh.share[tid][w] = ex2(moved + (sh.stats[w][tid][1] - scale));
                }
                if (whole) {                    // the segment's own: what is left to multiply by, and the logarithm
                    sh.share[tid][kTeamWarps] = out_factor<kFloat>(scale, total);
                    if (a.lse && block * kQueries + tid < a.group)
                        a.lse[(int64_t)sequence * a.shape.heads * a.group + head * a.group + block * kQueries + tid] =
                            total != 0.0f ? (r + log2f(total)) * 0.693147180559945309f : -INFINITY;
                } else {
                    *reinterpret_cast<float4*>(partials + slot * kPartial<P> + tid * (P + 4) + P) = make_float4(r, scale, total, 0.0f);
                }
            }
            team_sync(team);
            for (int i = tid; i < (kRests ? 4 : kQueries) * P / 4; i += kTeam) {
                const int query = i / (P / 4), d = (i % (P / 4)) * 4;
                const float* share = sh.share[query];
                float4 sum4 = make_float4(0, 0, 0, 0);
#pragma unroll
                for (int w = 0; w < kTeamWarps; ++w) {
                    float4 v = *reinterpret_cast<const float4*>(
                        reinterpret_cast<const float*>(shared + X::stages_at(team * kTeamWarps + w)) + ((query & 1) * 4 + (query >> 1)) * (P + 4) + d);
                    const float f = share[w];
                    if constexpr (kRestsBoth) {               // what the weights' rounding left, of query + 4
                        const float4 u = *reinterpret_cast<const float4*>(
                            reinterpret_cast<const float*>(shared + X::stages_at(team * kTeamWarps + w)) + ((query & 1) * 4 + (query >> 1) + 2) * (P + 4) + d);
                        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                    }
                    sum4.x += v.x * f; sum4.y += v.y * f; sum4.z += v.z * f; sum4.w += v.w * f;
                }
                if (whole) {
                    if (block * kQueries + query < a.group) {
                        const float f = share[kTeamWarps];
                        store_four<kFloat>(a.out, row_of(a.out, sequence, head * a.group + block * kQueries + query), d, a.shape.dim,
                                           make_float4(sum4.x * f, sum4.y * f, sum4.z * f, sum4.w * f));
                    }
                } else {
                    *reinterpret_cast<float4*>(partials + slot * kPartial<P> + query * (P + 4) + d) = sum4;
                }
            }
            if (starts && !whole && tid == 0) {
                // the team that has the segment's last unit: the largest one whose share begins at or before it
                const int64_t unit = at + ours - count + units - 1;
                Record rec;
                rec.sequence = sequence; rec.head_block = hb; rec.last = (int32_t)(((unit + 1) * parts - 1) / all); rec.pad = 0;
                records[me] = rec;
            }
            at += ours;
            chunk = -kStart;
            if (at < end && ++hb == head_blocks) {
                hb = 0;
                do { extent = extent_of(a, ++sequence); units = extent.template units<X::kUnit>(); } while (units == 0);
            }
            team_sync(team);                                            // the sums have been read
        }
    }

    // sequences without a token to see
    for (int b = me; b < a.batch; b += teams) {
        if (extent_of(a, b).template units<X::kUnit>() > 0) continue;
        const int queries = a.shape.heads * a.group;
        for (int64_t i = tid; i < (int64_t)queries * a.shape.dim; i += kTeam)
            store_any(a.out.type, row_of(a.out, b, (int)(i / a.shape.dim)), (int)(i % a.shape.dim), 0.0f);
        if (a.lse) for (int i = tid; i < queries; i += kTeam) a.lse[(int64_t)b * queries + i] = -INFINITY;
    }
}

// Joins the partial sums of a segment that began in team `blockIdx.x` and went on in others: kJoinWarps warps a query, each
// with a share of the teams, so that what has to be read is under way at once (one warp a query took 8 us for 37 teams).
constexpr int kJoinWarps = 4;
template <int P>
__global__ void __launch_bounds__(32 * kQueries* kJoinWarps) attend_join_kernel(const __grid_constant__ CacheAttendArgs a)
{
    constexpr int kVectors = P / 128 > 0 ? P / 128 : 1;                 // of 4 coordinates a lane
    __shared__ float4 sums[kJoinWarps][kQueries][kVectors][32];
    __shared__ float4 stats[kJoinWarps][kQueries];      // reference, scale of the weights, denominator
    pdl_wait();
    pdl_launch_next();
    const float* const workspace = fresh(a.partial);
    const Record rec = reinterpret_cast<const Record*>(workspace)[blockIdx.x];
    if (rec.sequence < 0) return;
    const int lane = threadIdx.x & 31, q = (threadIdx.x >> 5) % kQueries, share = (threadIdx.x >> 5) / kQueries, begin = blockIdx.x;
    const float* partials = workspace + (int64_t)gridDim.x * (sizeof(Record) / 4) + q * (P + 4);
    auto part = [&](int c) { return partials + (2 * (int64_t)c + (c == begin)) * kPartial<P>; };
    // four teams' partials are read at once where there are as many; reference and scale move with each group
    float r = kLow, scale = 0.0f, total = 0.0f;
    float4 acc[kVectors] = {};
    int c = begin + share;
    auto take = [&](auto teams) {
        constexpr int kTeams = decltype(teams)::value;
        float4 st[kTeams], v[kTeams][kVectors] = {};
#pragma unroll
        for (int j = 0; j < kTeams; ++j) {
            const float* p = part(c + kJoinWarps * j);
            st[j] = __ldcg(reinterpret_cast<const float4*>(p + P));
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
                if (P >= 128 || lane < P / 4) v[j][i] = __ldcg(reinterpret_cast<const float4*>(p + 4 * (lane + 32 * i)));
        }
        float r1 = r;
#pragma unroll
        for (int j = 0; j < kTeams; ++j) r1 = fmaxf(r1, st[j].x);
        const float here = r - r1;
        float scale1 = scale + here;
#pragma unroll
        for (int j = 0; j < kTeams; ++j) scale1 = fmaxf(scale1, st[j].y + (st[j].x - r1));
        scale1 = whole_scale(scale1);
        total *= ex2(here);
        const float old = ex2(here + (scale - scale1));
#pragma unroll
        for (int i = 0; i < kVectors; ++i) { acc[i].x *= old; acc[i].y *= old; acc[i].z *= old; acc[i].w *= old; }
#pragma unroll
        for (int j = 0; j < kTeams; ++j) {
            const float there = st[j].x - r1, f = ex2(there + (st[j].y - scale1));
            total += st[j].z * ex2(there);
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                acc[i].x += v[j][i].x * f; acc[i].y += v[j][i].y * f; acc[i].z += v[j][i].z * f; acc[i].w += v[j][i].w * f;
            }
        }
        r = r1; scale = scale1;
        c += kJoinWarps * kTeams;
    };
#pragma unroll 1
    while (c + 3 * kJoinWarps <= rec.last) take(std::integral_constant<int, 4>());
#pragma unroll 1
    while (c + kJoinWarps <= rec.last) take(std::integral_constant<int, 2>());
    if (c <= rec.last) take(std::integral_constant<int, 1>());
#pragma unroll
    for (int i = 0; i < kVectors; ++i) sums[share][q][i][lane] = acc[i];
    if (lane == 0) stats[share][q] = make_float4(r, scale, total, 0.0f);
    __syncthreads();
    const int head = rec.head_block / a.group_blocks, query = (rec.head_block - head * a.group_blocks) * kQueries + q;
    if (share > 0 || query >= a.group) return;
    for (int s = 1; s < kJoinWarps; ++s) r = fmaxf(r, stats[s][q].x);
    scale = -INFINITY;
    for (int s = 0; s < kJoinWarps; ++s) scale = fmaxf(scale, stats[s][q].y + (stats[s][q].x - r));
    scale = whole_scale(scale);
    float f[kJoinWarps];
    total = 0.0f;
#pragma unroll
    for (int s = 0; s < kJoinWarps; ++s) {
        const float moved = stats[s][q].x - r;
        total += stats[s][q].z * ex2(moved);
        f[s] = ex2(moved + (stats[s][q].y - scale));
    }
    const float out = a.out.type == LQ_F32 ? out_factor<true>(scale, total) : out_factor<false>(scale, total);
    char* const to = row_of(a.out, rec.sequence, head * a.group + query);
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
        float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int s = 0; s < kJoinWarps; ++s) {
            const float4 u = sums[s][q][i][lane];
            v.x += u.x * f[s]; v.y += u.y * f[s]; v.z += u.z * f[s]; v.w += u.w * f[s];
        }
        const float o[4] = {v.x * out, v.y * out, v.z * out, v.w * out};
        const int d = 4 * (lane + 32 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) if (d + k < a.shape.dim) store_any(a.out.type, to, d + k, o[k]);
    }
    if (lane == 0 && a.lse)
        a.lse[(int64_t)rec.sequence * a.shape.heads * a.group + head * a.group + query] =
            total != 0.0f ? (r + log2f(total)) * 0.693147180559945309f : -INFINITY;
}

template <int P, int WK, int WV, int kMode>
cudaError_t launch_as(const CacheAttendArgs& a, cudaStream_t s)
{
    using X = Stage<P, WK, WV>;
    constexpr int kBytes = smem_bytes<P, WK, WV>();
    static_assert(kBytes <= 227 << 10, "shared memory of an SM");
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = opt_in_shared_memory(configured, kBytes, attend_kernel<P, WK, WV, kMode>);
    if (e == cudaSuccess) e = lq::launch(attend_kernel<P, WK, WV, kMode>, a.sms, X::kTeams * kTeam, kBytes, s, a);
    if (e == cudaSuccess && a.partial) e = lq::launch(attend_join_kernel<P>, a.sms * X::kTeams, 32 * kQueries * kJoinWarps, 0, s, a);
    return e;
}

template <int P, int WK, int WV>
cudaError_t launch_mode(const CacheAttendArgs& a, cudaStream_t s)
{
    const bool beside = a.group <= 4;
    if (a.queries.type == LQ_F32) return beside ? launch_as<P, WK, WV, kBesideBoth>(a, s) : launch_as<P, WK, WV, kTwoBoth>(a, s);
    if (a.queries.type == LQ_F16) {
        if (beside) return launch_as<P, WK, WV, kBesideHalf>(a, s);
        return a.rotary.table ? launch_as<P, WK, WV, kTwoBothHalf>(a, s) : launch_as<P, WK, WV, kWeights>(a, s);
    }
    if (a.rotary.table) return beside ? launch_as<P, WK, WV, kBeside>(a, s) : launch_as<P, WK, WV, kTwo>(a, s);
    return launch_as<P, WK, WV, kPlain>(a, s);
}

template <int P>
cudaError_t launch(const CacheAttendArgs& a, cudaStream_t s)
{
    if (a.shape.sym_bits[0] == 4) return a.shape.sym_bits[1] == 4 ? launch_mode<P, 4, 4>(a, s) : launch_mode<P, 4, 8>(a, s);
    return a.shape.sym_bits[1] == 4 ? launch_mode<P, 8, 4>(a, s) : launch_mode<P, 8, 8>(a, s);
}

}  // namespace attend
}  // namespace lq
