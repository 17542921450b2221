// Attention of one new token a sequence over a prefix that all sequences of the batch share, the prefix read and decoded once for all.
//
// Mathematics: that of lq_cache_attend.cuh.  With c_j = (2^e q) . level(K_j) and f = scale log2(e) / 2^e
//   d_j = (c_j f) N_j - ref,  p_j = exp2(d_j),  w_j = p_j M_j 2^(6 - k),  out = 2^(k - 6) sum_j w_j level(V_j) / sum_j p_j,
// N and M the keys' and values' norms, ref a running reference of the scores and k a whole number, the running scale of the weights: both
// move, and the sums with them, only when a score passes its reference by 8 powers of two, or a weight its scale.  Scores, p, w and all
// sums are fp32.  Levels are fp16 as they stand.  Roundings to fewer bits: q as fp16 after a power of two (exact for fp16 and bf16;
// rotated and fp32 ones as a sum of two, 22 bits); w as fp16 for bf16 outputs (11 bits, an eighth of the output's own rounding), as a sum of
// two for fp16 and fp32 ones (22 bits).
//
// Work.  All sequences' queries of one head of the cache are the rows of a matrix, 128 of them a block: both products are dense, and
// run on tcgen05: S = Q K^T (128 x 64 tokens, Q and K in shared memory) and O += W V (W in tensor memory, where the scores stood; V in
// shared memory, tokens outermost).  What q's rounding left is a second operand in tensor memory, what w's left stands beside W.
// A CTA has two slots (one for rows of 256), each with scores, sums and four warps of its own, so that one slot's scores go through the
// softmax while the other's products run: two blocks of rows over the same tiles of 64 tokens or, where a block is alone, that
// block over even and odd tiles.  Eight warps decode: a byte of a row is looked up in a table of shared memory that has a copy in each lane's bank
// (as in lq_cache_attend.cuh), 8 coordinates are 16 bytes of a tile, swizzled by 128 bytes as the matrix unit reads it.
//
// Split.  The prefix's tiles of a (head, pair of blocks) are dealt to several CTAs such that the GPU is full; each leaves for every row its
// sums, reference, scale and denominator, and a second kernel joins them with those of the sequence's own tokens.
//
// Waits are bounded: after some two seconds a waiting thread sets LQ_CACHE_GAVE_UP, and all leave.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

namespace lq {
namespace {

constexpr int kRows = 128;              // rows of a block: lanes of tensor memory
constexpr int kTile = 64;               // tokens
constexpr int kDecodeWarps = 8, kDecode = 32 * kDecodeWarps;
constexpr int kTableAt = 1 << 16, kTableBytes = 256 * 256, kSystemBytes = 1 << 10;      // as in lq_cache_attend.cuh
constexpr int kHighAt = kTableAt + kTableBytes;
constexpr int kPanelQ = kRows * 128, kPanel = kTile * 128;      // bytes of 64 coordinates of a block's rows, of a tile's
constexpr float kLow = -3.402823466e38f;
constexpr float kSlack = 8.0f;
constexpr int kLift = 6;
constexpr int kColumns = 512;           // of tensor memory: all (one CTA an SM)

// Shared memory, by address.  Below the table: pieces (a tile's keys or values), then what is small; behind it: the queries, then pieces.
template <int P>
struct Layout {
    static constexpr int kSlots = cache_shared_slots(P), kPanels = P / 64, kPiece = P * 128;
    static constexpr int kStages = P == 256 ? 1 : 2;
    static constexpr int kThreads = 128 * kSlots + kDecode + 32;
    static constexpr int kDecodeAt = 4 * kSlots, kIssuer = kDecodeAt + kDecodeWarps;    // warps
    static constexpr int kQueries = kSlots * kPanels * kPanelQ;
    static constexpr int kLowPieces = P == 64 ? 4 : P == 128 ? 3 : 1;
    static constexpr int kSmallAt = kSystemBytes + kLowPieces * kPiece;
    static constexpr int kEnd = kHighAt + kQueries + (2 * kStages - kLowPieces) * kPiece;
    static __device__ __forceinline__ uint32_t piece(int i)     // 2 * stage + (0: keys, 1: values)
    {
        return i < kLowPieces ? kSystemBytes + i * kPiece : kHighAt + kQueries + (i - kLowPieces) * kPiece;
    }
    static __device__ __forceinline__ uint32_t queries(int slot, int panel) { return kHighAt + (slot * kPanels + panel) * kPanelQ; }
    // what the queries' rounding leaves, before it goes to tensor memory: in the pieces' place
    static __device__ __forceinline__ uint32_t rests(int slot, int panel)
    {
        const int at = (slot * kPanels + panel) * kPanelQ;
        return piece(at / kPiece) + at % kPiece;
    }
    // tensor memory, columns of a slot
    static constexpr int kScores = 0, kSums = kTile, kRests = kTile + P, kSlotColumns = kTile + P + P / 2;
    static_assert(kSlots * kSlotColumns <= kColumns && kEnd <= 227 << 10 && kSlots * kPanels * kPanelQ <= 2 * kStages * kPiece, "places");
};

struct Small {
    uint64_t full[2], empty[2];         // a stage holds a tile; has been read
    uint64_t scored[2], weighed[2], summed[2];          // of a slot: its scores are there, its weights, its sums
    uint64_t drained;
    uint32_t tensor;                    // address of tensor memory
    uint32_t failed;
    uint32_t seen[2][2];                // of a stage: bit per token
    int32_t exponent[2];                // of a stage: what the values' norms are divided by
    alignas(16) float keys[2][kTile];   // norms
    alignas(16) float values[2][kTile];
    float factor[2 * kRows];
};

// ---- instructions ----------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t address_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* b, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(address_of(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void arrive(uint64_t* b)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(address_of(b)) : "memory");
}
__device__ __forceinline__ bool passed(uint64_t* b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(address_of(b)), "r"(parity) : "memory");
    return ok;
}
// False after some two seconds, or once another thread has given up.
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, Small& sm, uint32_t* flags)
{
    if (passed(b, parity)) return true;
    const long long start = clock64();
    while (!passed(b, parity)) {
        if (*reinterpret_cast<volatile uint32_t*>(&sm.failed)) return false;
        if (clock64() - start > 1ll << 32) {
            *reinterpret_cast<volatile uint32_t*>(&sm.failed) = 1;
            atomicOr(flags, LQ_CACHE_GAVE_UP);
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* b)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(address_of(b)) : "memory");
}

// 32 columns of this warp's 32 lanes.
__device__ __forceinline__ void tensor_load32(uint32_t (&v)[32], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
                   "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
                   "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_store32(uint32_t at, const uint32_t (&v)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                    "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]),
                    "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]),
                    "r"(v[30]), "r"(v[31])
                 : "memory");
}

// Operand in shared memory, swizzled by 128 bytes.  K along the rows of 128 bytes: rows in groups of 8, 1024 bytes apart.  N along them
// (tokens outermost): the next 64 coordinates are a panel further, the next 8 tokens 1024 bytes.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading)
{
    return (uint64_t)((at >> 4) & 0x3fff) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp16 operands, fp32 sums
__host__ __device__ constexpr uint32_t instruction(int n, bool n_outermost) { return 1u << 4 | (uint32_t)n_outermost << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRows >> 4) << 24; }

__device__ __forceinline__ void multiply(uint32_t sums, uint64_t a, uint64_t b, uint32_t how, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(sums), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void multiply_tensor(uint32_t sums, uint32_t a, uint64_t b, uint32_t how, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(sums), "r"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }        // -126 .. 127
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 255) - 127; }

__device__ __forceinline__ uint32_t halves(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const uint32_t&>(h);
}
__device__ __forceinline__ uint32_t rest_of(uint32_t rounded, float lo, float hi)
{
    const float2 r = __half22float2(reinterpret_cast<const __half2&>(rounded));
    return halves(lo - r.x, hi - r.y);
}

template <int kByte>
__device__ __forceinline__ uint32_t look(uint32_t w, uint32_t lane_base)
{
    uint32_t v;
    asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(__byte_perm(w, lane_base, 0x7604 | (kByte << 4))));
    return v;
}
__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void store2(uint32_t at, __half v)
{
    asm volatile("st.shared.b16 [%0], %1;" :: "r"(at), "h"(__half_as_ushort(v)) : "memory");
}

// Where coordinate d of row r stands in a panel of rows of 128 bytes.
__device__ __forceinline__ uint32_t swizzled(int r, int chunk) { return (uint32_t)(r * 128 + ((chunk ^ (r & 7)) << 4)); }

// ---- a CTA's share ---------------------------------------------------------------------------------------------

struct Share {
    int head, block;                    // of the cache; first block of rows
    int tile0, tiles;                   // its tiles of the prefix
    int64_t length;                     // of the prefix
    bool pair;                          // two blocks of rows; else (two slots) even and odd tiles
};

template <int P>
__device__ __forceinline__ Share share_of(const CacheSharedArgs& a)
{
    constexpr int kSlots = cache_shared_slots(P);
    Share s;
    const int blocks = (int)(((int64_t)a.batch * a.group + kRows - 1) / kRows), pairs = (blocks + kSlots - 1) / kSlots;
    const int split = blockIdx.x % a.splits, item = blockIdx.x / a.splits;
    s.head = item / pairs;
    s.block = (item - s.head * pairs) * kSlots;
    s.pair = kSlots == 2 && s.block + 1 < blocks;
    const int given = *a.prefix_length;
    s.length = given < 0 ? 0 : given > a.prefix_most ? a.prefix_most : given;
    if (given != s.length && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
    const int64_t all = (s.length + kTile - 1) / kTile;
    s.tile0 = (int)(all * split / a.splits);
    s.tiles = (int)(all * (split + 1) / a.splits) - s.tile0;
    return s;
}

// Row `row` of a head: query row % group of sequence row / group.  A warp brings it into shared memory: times its power of two, as fp16 and the rest.
template <int P>
__device__ __forceinline__ void bring_query(const CacheSharedArgs& a, const Share& s, Small& sm, int slot, int place, int lane)
{
    using L = Layout<P>;
    const int64_t row = (int64_t)(s.block + slot) * kRows + place;
    const bool live = row < (int64_t)a.batch * a.group;
    float x[P / 32];
    bool lost = false;
#pragma unroll
    for (int i = 0; i < P / 32; ++i) x[i] = 0.0f;
    if (live) {
        const int sequence = (int)(row / a.group), query = (int)(row - (int64_t)sequence * a.group);
        const char* from = static_cast<const char*>(a.queries.data) + (int64_t)sequence * a.queries.token_bytes +
                           (int64_t)(s.head * a.group + query) * a.queries.head_bytes;
        auto number = [&](int d) -> float {
            if (a.queries.type == LQ_F32) return reinterpret_cast<const float*>(from)[d];
            if (a.queries.type == LQ_F16) return __half2float(reinterpret_cast<const __half*>(from)[d]);
            return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(from)[d]);
        };
        const CacheRotary& r = a.rotary;
        const float* angles = r.table;
        if (r.table) {
            int64_t at;
            if (r.at) {
                at = r.at[sequence];
            } else {
                const int n = a.lengths[sequence];
                const int64_t last = s.length + (n < 0 ? 0 : n > a.own_most ? a.own_most : n);
                at = last > 0 ? last - 1 : 0;
            }
            lost = at < 0 || at >= r.positions;
            if (lost) { if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION); }
            else angles += at * r.dim;
        }
        const int half = r.dim / 2;
#pragma unroll
        for (int i = 0; i < P / 32; ++i) {
            const int d = lane + 32 * i;
            x[i] = d < a.shape.dim ? number(d) : 0.0f;
            if (r.table && !lost && d < r.dim) {
                const bool lower = r.interleaved ? d % 2 == 0 : d < half;
                const int p = r.interleaved ? d / 2 : d < half ? d : d - half;
                const float u = number(r.interleaved ? d ^ 1 : lower ? d + half : d - half), c = angles[p], t = angles[half + p];
                x[i] = lower ? __fsub_rn(__fmul_rn(x[i], c), __fmul_rn(u, t)) : __fadd_rn(__fmul_rn(x[i], c), __fmul_rn(u, t));
            }
            if (lost) x[i] = __uint_as_float(0x7fffffffu);
        }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < P / 32; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    // 2^e brings the largest coordinate to [2^14, 2^15); Inf and NaN stay what they are
    const int e = min(top >= 0x7f800000u || top == 0 ? 0 : 141 - (int)(top >> 23), 120);
#pragma unroll
    for (int i = 0; i < P / 32; ++i) {
        const int d = lane + 32 * i;
        const float y = x[i] * power(e);
        const __half h = __float2half_rn(y);
        const uint32_t at = swizzled(place, (d & 63) >> 3) + (d & 7) * 2;
        store2(L::queries(slot, d >> 6) + at, h);
        if (a.two_queries) store2(L::rests(slot, d >> 6) + at, __float2half_rn(y - __half2float(h)));
    }
    if (lane == 0) sm.factor[slot * kRows + place] = a.scale * power(-e);
}

// ---- decoding --------------------------------------------------------------------------------------------------

// Symbols of 8 coordinates of a thread's rows of a tile, and what one warp brings of its norms.
template <int P>
struct Codes {
    static constexpr int kEach = kTile * (P / 8) / kDecode;     // rows (of keys, and of values) that a thread has 8 coordinates of
    uint2 w[2][kEach];
    float keys[2], values[2];
    uint32_t seen;                      // bit i: the tile's i-th 16 tokens are on a page that is there
};

// The page of 16 of a tile's tokens, by lanes 0 to 3; -1 past the end.
__device__ __forceinline__ int page_of(const CacheSharedArgs& a, const Share& s, int tile, bool inside, int lane)
{
    const int64_t token = (int64_t)(s.tile0 + tile) * kTile + 16 * lane;
    if (!inside || lane >= kTile / 16 || token >= s.length) return -1;
    const int page = a.prefix[token >> a.shape.page_shift];
    if (page < 0 || page >= a.num_pages) {
        atomicOr(a.flags, LQ_CACHE_BAD_PAGE);
        return -1;
    }
    return page;
}

template <int P>
__device__ __forceinline__ void fetch(Codes<P>& c, const CacheSharedArgs& a, const Share& s, int tile, int page, int tid)
{
    const int lane = tid & 31, mask = (1 << a.shape.page_shift) - 1;
    const int64_t first = (int64_t)(s.tile0 + tile) * kTile;
    c.seen = __ballot_sync(0xffffffffu, page >= 0) & 15u;
    const uint32_t values_at = (uint32_t)a.shape.row_words[0] << a.shape.page_shift, norms_at = values_at + ((uint32_t)a.shape.row_words[1] << a.shape.page_shift);
    auto head_of = [&](int p) { return a.pages + (int64_t)p * a.shape.page_words + (int64_t)s.head * a.shape.head_words; };
#pragma unroll
    for (int k = 0; k < Codes<P>::kEach; ++k) {
        const int unit = tid + kDecode * k, token = unit / (P / 8), col = unit % (P / 8);
        const int p = __shfl_sync(0xffffffffu, page, token >> 4);
        c.w[0][k] = c.w[1][k] = make_uint2(0, 0);
        if (p >= 0) {
            const uint32_t* base = head_of(p);
            const int row = (int)((first + token) & mask);
            const uint32_t* keys = base + row * a.shape.row_words[0];
            const uint32_t* values = base + values_at + row * a.shape.row_words[1];
            if (a.shape.sym_bits[0] == 8) c.w[0][k] = reinterpret_cast<const uint2*>(keys)[col]; else c.w[0][k].x = keys[col];
            if (a.shape.sym_bits[1] == 8) c.w[1][k] = reinterpret_cast<const uint2*>(values)[col]; else c.w[1][k].x = values[col];
        }
    }
    if (tid < 32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = lane + 32 * i, p = __shfl_sync(0xffffffffu, page, token >> 4);
            c.keys[i] = c.values[i] = 0.0f;
            if (p >= 0) {
                const float* norms = reinterpret_cast<const float*>(head_of(p) + norms_at) + ((first + token) & mask);
                c.keys[i] = norms[0];
                c.values[i] = norms[mask + 1];
            }
        }
    }
}

template <int P>
__device__ __forceinline__ void decode(const Codes<P>& c, const CacheSharedArgs& a, const Share& s, Small& sm, int tile, int stage, int tid)
{
    using L = Layout<P>;
    const int lane = tid & 31;
    const uint32_t base = kTableAt + 4 * lane;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        const uint32_t piece = L::piece(2 * stage + kind), copies = base + 128 * kind;
        const bool fine = a.shape.sym_bits[kind] == 8;
#pragma unroll
        for (int k = 0; k < Codes<P>::kEach; ++k) {
            const int unit = tid + kDecode * k, token = unit / (P / 8), col = unit % (P / 8);
            const uint2 w = c.w[kind][k];
            uint32_t v[4];
            if (fine) {
                auto two = [](uint32_t x, uint32_t y) { return __byte_perm(x, y, 0x5410); };
                v[0] = two(look<0>(w.x, copies), look<1>(w.x, copies)); v[1] = two(look<2>(w.x, copies), look<3>(w.x, copies));
                v[2] = two(look<0>(w.y, copies), look<1>(w.y, copies)); v[3] = two(look<2>(w.y, copies), look<3>(w.y, copies));
            } else {
                v[0] = look<0>(w.x, copies); v[1] = look<1>(w.x, copies); v[2] = look<2>(w.x, copies); v[3] = look<3>(w.x, copies);
            }
            store16(piece + (col >> 3) * kPanel + swizzled(token, col & 7), v[0], v[1], v[2], v[3]);
        }
    }
    if (tid < 32) {
        const int64_t first = (int64_t)(s.tile0 + tile) * kTile;
        uint32_t seen[2];
        int most = -127;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = lane + 32 * i;
            const bool there = (c.seen >> (token >> 4) & 1) && first + token < s.length;
            seen[i] = __ballot_sync(0xffffffffu, there);
            if (there) most = max(most, exponent_of(c.values[i]));
        }
        most = __reduce_max_sync(0xffffffffu, most);
        const int half = most / 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = lane + 32 * i;
            const bool there = seen[i] >> lane & 1;
            sm.keys[stage][token] = there ? c.keys[i] : 0.0f;
            sm.values[stage][token] = there ? c.values[i] * power(-half) * power(half - most) : 0.0f;
        }
        if (lane == 0) { sm.seen[stage][0] = seen[0]; sm.seen[stage][1] = seen[1]; sm.exponent[stage] = most; }
    }
}

// ---- softmax ---------------------------------------------------------------------------------------------------

// One row's running state.
struct Row {
    float f;                            // of the scores
    float ref = 0.0f, total = 0.0f;
    int scale = 0;
    bool begun = false;
};

__device__ __forceinline__ uint64_t pair_of(float x, float y) { uint64_t v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y)); return v; }
__device__ __forceinline__ void parted(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t v; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b)); return v; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t v; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b)); return v; }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}

// The scores of a tile become weights, in their place.  `sums`: this slot's, moved where reference or scale moves; `none`: there are none yet.
template <int P, bool kTwo>
__device__ __forceinline__ void weigh_tile(Row& row, const Small& sm, int stage, uint32_t scores, uint32_t sums, bool none)
{
    float d[kTile];
    {
        uint32_t (&lo)[32] = *reinterpret_cast<uint32_t (*)[32]>(&d[0]);
        uint32_t (&hi)[32] = *reinterpret_cast<uint32_t (*)[32]>(&d[32]);
        tensor_load32(lo, scores);
        tensor_load32(hi, scores + 32);
        loaded();
    }
    const uint64_t f2 = pair_of(row.f, row.f), minus = pair_of(-row.ref, -row.ref);
#pragma unroll
    for (int j = 0; j < kTile; j += 4) {
        const float4 n = *reinterpret_cast<const float4*>(&sm.keys[stage][j]);
        parted(fma2(mul2(pair_of(d[j], d[j + 1]), f2), pair_of(n.x, n.y), minus), d[j], d[j + 1]);
        parted(fma2(mul2(pair_of(d[j + 2], d[j + 3]), f2), pair_of(n.z, n.w), minus), d[j + 2], d[j + 3]);
    }
    const uint32_t seen0 = sm.seen[stage][0], seen1 = sm.seen[stage][1];
    if ((seen0 & seen1) != 0xffffffffu) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (!(seen0 >> j & 1)) d[j] = -INFINITY;
            if (!(seen1 >> j & 1)) d[32 + j] = -INFINITY;
        }
    }
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < kTile; j += 8)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = fmaxf(top[i], fmaxf(d[j + i], d[j + 4 + i]));
    const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    float moved = 0.0f;
    if (__any_sync(0xffffffffu, most > kSlack || !row.begun)) {
        const float step = row.begun ? fmaxf(most, 0.0f) : most;
        if (step > -INFINITY) {
            const float ref = row.ref + step;
            moved = row.ref - ref;
            row.ref = ref;
#pragma unroll
            for (int j = 0; j < kTile; ++j) d[j] += moved;
            if (row.begun) row.total *= ex2(moved);
        }
    }
    uint64_t total[2] = {0, 0};
    float heavy[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kTile; j += 4) {
        const float4 m = *reinterpret_cast<const float4*>(&sm.values[stage][j]);
        const uint64_t p = pair_of(ex2(d[j]), ex2(d[j + 1])), q = pair_of(ex2(d[j + 2]), ex2(d[j + 3]));
        total[0] = add2(total[0], p);
        total[1] = add2(total[1], q);
        parted(mul2(p, pair_of(m.x, m.y)), d[j], d[j + 1]);
        parted(mul2(q, pair_of(m.z, m.w)), d[j + 2], d[j + 3]);
        heavy[0] = fmaxf(heavy[0], fmaxf(d[j], d[j + 1]));
        heavy[1] = fmaxf(heavy[1], fmaxf(d[j + 2], d[j + 3]));
    }
    {
        float x, y;
        parted(add2(total[0], total[1]), x, y);
        row.total += x + y;
    }
    // the largest weight is 2^(exponent + e) or twice that
    const int exponent = sm.exponent[stage], e = exponent_of(fmaxf(heavy[0], heavy[1]));
    const bool over = exponent + e >= row.scale + (int)kSlack || exponent - row.scale > 114 || !row.begun;
    if (__any_sync(0xffffffffu, over || moved != 0.0f)) {
        // (an exponent's difference is whole but for `moved`, whose fraction the scale's rounding down leaves to the factor)
        float factor = 1.0f;
        if (over || moved != 0.0f) {
            int scale = max(exponent + e, exponent - 114);
            if (row.begun) scale = max(scale, (int)floorf(fmaxf((float)row.scale + moved, -1000.0f)));
            factor = row.begun ? ex2(moved + (float)(row.scale - scale)) : 0.0f;
            row.scale = scale;
            row.begun = row.begun || most > -INFINITY;
        }
        if (!none) {
#pragma unroll 1
            for (int c = 0; c < P; c += 32) {
                uint32_t v[32];
                tensor_load32(v, sums + c);
                loaded();
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * factor);
                tensor_store32(sums + c, v);
            }
        }
    }
    const float lift = power(max(-126, min(127, exponent - row.scale + kLift)));
    const uint64_t lift2 = pair_of(lift, lift);
    uint32_t w[32];
    uint32_t rest[kTwo ? 32 : 1];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        float x, y;
        parted(mul2(pair_of(d[2 * j], d[2 * j + 1]), lift2), x, y);
        w[j] = halves(x, y);
        if constexpr (kTwo) rest[j] = rest_of(w[j], x, y);
    }
    tensor_store32(scores, w);
    if constexpr (kTwo) tensor_store32(scores + 32, rest);
    stored();
}

// ---- the kernel ------------------------------------------------------------------------------------------------

template <int P, bool kTwo>
__global__ void __launch_bounds__(Layout<P>::kThreads, 1) shared_prefix_kernel(const __grid_constant__ CacheSharedArgs a)
{
    using L = Layout<P>;
    extern __shared__ __align__(1024) char smem[];
    char* const shared = smem - __cvta_generic_to_shared(smem);         // shared address 0
    Small& sm = *reinterpret_cast<Small*>(shared + L::kSmallAt);
    static_assert(L::kSmallAt + sizeof(Small) <= kTableAt, "below the table");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    for (int i = tid; i < 512; i += L::kThreads) {                      // the look-up table: half an entry's row each
        const uint32_t v = a.tables[i & 1].pairs[i >> 1];
        uint4* row = reinterpret_cast<uint4*>(shared + kTableAt + i * 128);
#pragma unroll
        for (int j = 0; j < 8; ++j) row[(j + lane) & 7] = make_uint4(v, v, v, v);
    }
    if (warp == L::kIssuer) {
        if (lane == 0) {
            for (int i = 0; i < 2; ++i) {
                barrier_init(&sm.full[i], kDecode); barrier_init(&sm.empty[i], 1);
                barrier_init(&sm.scored[i], 1); barrier_init(&sm.weighed[i], 128); barrier_init(&sm.summed[i], 1);
            }
            barrier_init(&sm.drained, 1);
            sm.failed = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(address_of(&sm.tensor)), "n"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    pdl_wait();
    pdl_launch_next();
    const Share s = share_of<P>(a);
    const int rows = s.pair ? 2 * kRows : kRows;
    for (int r = warp; r < rows; r += L::kThreads / 32) bring_query<P>(a, s, sm, r / kRows, r % kRows, lane);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tensor = sm.tensor;
    // slot s of a use: pairs of blocks take every tile twice
    const int slots = L::kSlots, uses = s.pair ? 2 * s.tiles : s.tiles;
    auto tile_of = [&](int use) { return s.pair ? use >> 1 : use; };

    const int slot = warp >> 2;                                         // (of the softmax's warps)
    const int64_t my_row = (int64_t)(s.block + (s.pair ? slot : 0)) * kRows + (tid & 127);
    const uint32_t lanes = tensor + ((uint32_t)(32 * (warp & 3)) << 16), mine = lanes + slot * L::kSlotColumns;
    if (warp < L::kDecodeAt && a.two_queries) {                         // what the queries' rounding left goes to tensor memory
        const int from = s.pair ? slot : 0, r = tid & 127;
#pragma unroll 1
        for (int p = 0; p < L::kPanels; ++p) {
            uint32_t v[32];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint4 x = *reinterpret_cast<const uint4*>(shared + L::rests(from, p) + swizzled(r, c));
                v[4 * c] = x.x; v[4 * c + 1] = x.y; v[4 * c + 2] = x.z; v[4 * c + 3] = x.w;
            }
            tensor_store32(mine + L::kRests + 32 * p, v);
        }
        stored();
        fence_before();
    }
    if (a.two_queries) {
        __syncthreads();
        fence_after();
    }

    if (warp < L::kDecodeAt) {
        // ---- softmax: a thread has a row
        Row row;
        row.f = sm.factor[(s.pair ? slot : 0) * kRows + (tid & 127)];
        const bool live = __any_sync(0xffffffffu, my_row < (int64_t)a.batch * a.group);
        int n = 0;
        bool ok = true;
        for (int use = slot; use < uses && ok; use += slots, ++n) {
            const int tile = tile_of(use), stage = tile % L::kStages;
            ok = wait(&sm.full[stage], (tile / L::kStages) & 1, sm, a.flags) && wait(&sm.scored[slot], n & 1, sm, a.flags);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            if (live) weigh_tile<P, kTwo>(row, sm, stage, mine + L::kScores, mine + L::kSums, n == 0);
            fence_before();
            arrive(&sm.weighed[slot]);
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, wait(&sm.summed[slot], (n - 1) & 1, sm, a.flags));
        fence_after();
        if (live) {
            // ---- what is left of this row; of a block that is alone, one part of even tiles and one of odd ones
            const int part = blockIdx.x % a.splits + (slot == 1 && !s.pair ? a.splits : 0);
            const int64_t all_rows = (int64_t)a.batch * a.shape.heads * a.group;
            const int sequence = (int)(my_row / a.group);
            const bool there = my_row < (int64_t)a.batch * a.group;
            float* const to = a.parts + (part * all_rows + (int64_t)sequence * a.shape.heads * a.group + s.head * a.group +
                                         (my_row - (int64_t)sequence * a.group)) * cache_part_floats(P);
            if (n > 0 && ok) {
#pragma unroll 1
                for (int c = 0; c < P; c += 32) {
                    uint32_t v[32];
                    tensor_load32(v, mine + L::kSums + c);
                    loaded();
                    if (there)
#pragma unroll
                        for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(to + c + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
            if (there)
                *reinterpret_cast<float4*>(to + P) = make_float4(row.begun ? row.ref : kLow, (float)(row.scale - kLift), n > 0 && ok ? row.total : 0.0f, 0.0f);
        }
        fence_before();
    } else if (warp < L::kIssuer) {
        // ---- decoding: codes a tile ahead, pages two
        const int t = tid - 32 * L::kDecodeAt;
        Codes<P> codes;
        int page = page_of(a, s, 0, s.tiles > 0, lane);
        if (s.tiles > 0) fetch<P>(codes, a, s, 0, page, t);
        page = page_of(a, s, 1, s.tiles > 1, lane);
        for (int tile = 0; tile < s.tiles; ++tile) {
            const int stage = tile % L::kStages;
            const Codes<P> now = codes;
            if (tile + 1 < s.tiles) fetch<P>(codes, a, s, tile + 1, page, t);
            page = page_of(a, s, tile + 2, tile + 2 < s.tiles, lane);
            if (!__all_sync(0xffffffffu, wait(&sm.empty[stage], (tile / L::kStages & 1) ^ 1, sm, a.flags))) break;
            decode<P>(now, a, s, sm, tile, stage, t);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            arrive(&sm.full[stage]);
        }
    } else if (lane == 0) {
        // ---- the products, by one thread
        bool ok = true;
        for (int v = 0; v < uses + slots && ok; ++v) {
            if (v >= slots) {
                const int use = v - slots, w = use % slots, tile = tile_of(use), stage = tile % L::kStages;
                ok = wait(&sm.weighed[w], (use / slots) & 1, sm, a.flags);
                if (!ok) break;
                fence_after();
                const uint32_t at = tensor + w * L::kSlotColumns, values = L::piece(2 * stage + 1);
                constexpr uint32_t how = instruction(P, true);
#pragma unroll
                for (int rest = 0; rest < (kTwo ? 2 : 1); ++rest)
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k)
                        multiply_tensor(at + L::kSums, at + L::kScores + 32 * rest + 8 * k, operand(values + k * 2048, kPanel), how,
                                        use >= slots || rest > 0 || k > 0);
                commit(&sm.summed[w]);
                if (!s.pair || w == slots - 1) commit(&sm.empty[stage]);
            }
            if (v < uses) {
                const int w = v % slots, tile = tile_of(v), stage = tile % L::kStages;
                ok = wait(&sm.full[stage], (tile / L::kStages) & 1, sm, a.flags);
                if (ok && v >= slots) ok = wait(&sm.summed[w], (v / slots - 1) & 1, sm, a.flags);       // (weights stand where the scores come)
                if (!ok) break;
                fence_after();
                const uint32_t at = tensor + w * L::kSlotColumns, keys = L::piece(2 * stage);
                constexpr uint32_t how = instruction(kTile, false);
                // (the rests first: each step cuts the sum's last bit off, which is worth nothing while the sum is small)
                if (a.two_queries)
#pragma unroll
                    for (int k = 0; k < P / 16; ++k)
                        multiply_tensor(at + L::kScores, at + L::kRests + 8 * k, operand(keys + k / 4 * kPanel + (k % 4) * 32, 16), how, k > 0);
#pragma unroll
                for (int k = 0; k < P / 16; ++k)
                    multiply(at + L::kScores, operand(L::queries(s.pair ? w : 0, k / 4) + (k % 4) * 32, 16), operand(keys + k / 4 * kPanel + (k % 4) * 32, 16),
                             how, a.two_queries || k > 0);
                commit(&sm.scored[w]);
            }
        }
        if (!ok) {                                                      // what is under way ends before tensor memory is given back
            commit(&sm.drained);
            const long long start = clock64();
            while (!passed(&sm.drained, 0) && clock64() - start < 1ll << 32) {}
        }
    }
    __syncthreads();
    if (warp == L::kIssuer) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tensor), "n"(kColumns));
    }
}

// ---- the join --------------------------------------------------------------------------------------------------

// A warp for a row: what its parts of the prefix and of its own tokens give, in their order.
constexpr int kJoinThreads = 128;

template <int P>
__global__ void __launch_bounds__(kJoinThreads) shared_join_kernel(const __grid_constant__ CacheSharedArgs a)
{
    constexpr int kVectors = P / 128 > 0 ? P / 128 : 1;
    pdl_wait();
    pdl_launch_next();
    const int lane = threadIdx.x & 31;
    const int64_t all_rows = (int64_t)a.batch * a.shape.heads * a.group, row = (int64_t)blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
    if (row >= all_rows) return;
    const int heads = a.shape.heads * a.group, sequence = (int)(row / heads), head = (int)(row - (int64_t)sequence * heads);
    const int64_t in_head = (int64_t)sequence * a.group + head % a.group;
    const int blocks = (int)(((int64_t)a.batch * a.group + kRows - 1) / kRows), block = (int)(in_head / kRows);
    const bool alone = cache_shared_slots(P) == 2 && blocks % 2 == 1 && block == blocks - 1;
    const int before = a.splits * (alone ? 2 : 1), parts = before + (a.own_most > 0 && a.lengths[sequence] > 0);
    const float* const prefix = fresh(a.parts);
    const float* const own = fresh(a.own);
    auto part = [&](int i) { return (i < before ? prefix + (i * all_rows + row) * cache_part_floats(P) : own + row * cache_part_floats(P)); };
    auto stats = [&](int i) { return __ldcg(reinterpret_cast<const float4*>(part(i) + P)); };
    float r = kLow, scale = -1000.0f, total = 0.0f;
    for (int i = lane; i < parts; i += 32) r = fmaxf(r, stats(i).x);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) r = fmaxf(r, __shfl_xor_sync(0xffffffffu, r, o));
    for (int i = lane; i < parts; i += 32) {
        const float4 t = stats(i);
        if (t.z != 0.0f) scale = fmaxf(scale, t.y + (t.x - r));
        total += t.z * ex2(t.x - r);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        scale = fmaxf(scale, __shfl_xor_sync(0xffffffffu, scale, o));
        total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    scale = floorf(scale);
    float4 acc[kVectors] = {};
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
        const float4 t = stats(i);
        if (t.z == 0.0f) continue;                              // (nothing seen, and nothing written)
        const float f = ex2((t.x - r) + (t.y - scale));
#pragma unroll
        for (int k = 0; k < kVectors; ++k)
            if (P >= 128 || lane < P / 4) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(part(i) + 4 * (lane + 32 * k)));
                acc[k].x += v.x * f; acc[k].y += v.y * f; acc[k].z += v.z * f; acc[k].w += v.w * f;
            }
    }
    // 2^scale / total, the power in two factors that are normal numbers
    const int n = min(max((int)scale, -252), 254), half = n >> 1;
    const float out = total != 0.0f ? 1.0f / total * power(half) * power(n - half) : 0.0f;
    char* const to = static_cast<char*>(a.out.data) + (int64_t)sequence * a.out.token_bytes + (int64_t)head * a.out.head_bytes;
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const float o[4] = {acc[k].x * out, acc[k].y * out, acc[k].z * out, acc[k].w * out};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 4 * (lane + 32 * k) + i;
            if (d >= a.shape.dim) break;
            if (a.out.type == LQ_F32) reinterpret_cast<float*>(to)[d] = o[i];
            else if (a.out.type == LQ_F16) reinterpret_cast<__half*>(to)[d] = __float2half_rn(o[i]);
            else reinterpret_cast<__nv_bfloat16*>(to)[d] = __float2bfloat16_rn(o[i]);
        }
    }
    if (lane == 0 && a.lse) a.lse[row] = total != 0.0f ? (r + log2f(total)) * 0.693147180559945309f : -INFINITY;
}

template <int P, bool kTwo>
cudaError_t launch_prefix(const CacheSharedArgs& a, cudaStream_t s)
{
    using L = Layout<P>;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = opt_in_shared_memory(configured, L::kEnd, shared_prefix_kernel<P, kTwo>);
    const int64_t blocks = ((int64_t)a.batch * a.group + kRows - 1) / kRows, items = a.shape.heads * ((blocks + L::kSlots - 1) / L::kSlots);
    if (e == cudaSuccess) e = launch(shared_prefix_kernel<P, kTwo>, (unsigned)(items * a.splits), L::kThreads, L::kEnd, s, a);
    return e;
}

template <int P>
cudaError_t launch_join(const CacheSharedArgs& a, cudaStream_t s)
{
    const int64_t rows = (int64_t)a.batch * a.shape.heads * a.group;
    return launch(shared_join_kernel<P>, (unsigned)((rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32)), kJoinThreads, 0, s, a);
}

}  // namespace

int cache_shared_splits(const CacheShape& shape, int64_t rows, int64_t prefix_tokens, bool exact, int sms)
{
    const int slots = cache_shared_slots(shape.padded);
    const int64_t blocks = (rows + kRows - 1) / kRows, items = shape.heads * ((blocks + slots - 1) / slots), tiles = (prefix_tokens + kTile - 1) / kTile;
    if (tiles == 0) return 0;
    // a tile of two blocks takes twice as long as one of a block alone; what a CTA takes besides is some 8 of those
    const int64_t each = blocks > 1 && slots == 2 ? 2 : 1;
    // fp32 outputs: sums of 1024 tokens at most, as the matrix unit cuts off what a sum's last bit does not hold
    int64_t best = 1, cost = INT64_MAX;
    for (int64_t n = exact ? (tiles + 15) / 16 : 1; n <= tiles; ++n) {
        const int64_t c = (items * n + sms - 1) / sms * ((tiles + n - 1) / n * each + 8);
        if (c < cost) { cost = c; best = n; }
        if (n >= 64 && n * items > 2 * sms) break;
    }
    return (int)best;
}

cudaError_t launch_cache_shared_prefix(const CacheSharedArgs& a, cudaStream_t s)
{
    const bool two = a.queries.type != LQ_BF16;
    if (a.shape.padded == 64) return two ? launch_prefix<64, true>(a, s) : launch_prefix<64, false>(a, s);
    if (a.shape.padded == 128) return two ? launch_prefix<128, true>(a, s) : launch_prefix<128, false>(a, s);
    return two ? launch_prefix<256, true>(a, s) : launch_prefix<256, false>(a, s);
}

cudaError_t launch_cache_shared_join(const CacheSharedArgs& a, cudaStream_t s)
{
    return a.shape.padded == 64 ? launch_join<64>(a, s) : a.shape.padded == 128 ? launch_join<128>(a, s) : launch_join<256>(a, s);
}

}  // namespace lq
