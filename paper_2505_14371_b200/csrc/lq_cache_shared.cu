// Attention of one new token a sequence over a prefix that all sequences of the batch share, the prefix read and decoded once for all.
//
// Mathematics: that of lq_cache_attend.cuh.  With c_j = (2^e q) . level(K_j) and f = scale log2(e) / 2^e
//   d_j = (c_j f) N_j - ref,  p_j = exp2(d_j),  w_j = p_j M_j 2^(6 - k),  out = 2^(k - 6) sum_j w_j level(V_j) / sum_j p_j,
// N and M the keys' and values' norms, ref and k whole numbers, the running reference of the scores and the running scale of the weights: both
// move, and the sums with them (by powers of two), only when p add up to 2^16 or a weight passes 2^14.  Scores, p, w and all
// sums are fp32.  Levels are fp16 as they stand.  Roundings to fewer bits: q as fp16 after a power of two (exact for fp16 and bf16;
// rotated and fp32 ones as a sum of two, 22 bits); w as fp16 for bf16 outputs (11 bits, an eighth of the output's own rounding), as a sum of
// two for fp16 and fp32 ones (22 bits).
//
// Work.  All sequences' queries of one head of the cache are the rows of a matrix, 128 of them a block: both products are dense, and
// run on tcgen05: S = Q K^T (128 x 64 tokens, Q and K in shared memory) and O += W V (W in tensor memory; V in shared memory, tokens
// outermost).  What the queries' rounding left is a second operand of the first product, in tensor memory; what the weights' left is one of the second.
// Tensor memory holds two slots, each with scores, weights, sums and four warps of softmax (one slot where that takes more than half: rows
// of 256, and rows of 128 with both rests).  A CTA takes two blocks of rows over the same tiles or, where a block is alone, one
// block whose even tiles go to one slot and whose odd ones to the other; the two then share the rests of rows of 128, which leave no room else.  The scores of a tile are made while the softmax of the one before
// runs: a slot's scores may come again once they have been taken to registers, its weights once the sums have them.
// Eight warps decode: a byte of a row is looked up in a table of shared memory that has a copy in each lane's bank (as in lq_cache_attend.cuh), a
// thread writes 64 coordinates of a token, swizzled by 128 bytes as the matrix unit reads them.  Two warps a slot issue products, so that each waits only for what
// its own need.
//
// Split.  The prefix's tiles of a (head, block or pair of blocks) are dealt to several CTAs such that the GPU is full; each leaves for every row its
// sums, reference, scale and denominator.  The sequences' own tokens go through lq_cache_attend's kernel, which leaves the same, and a last kernel joins them.
//
// What bounds it: the softmax.  Of a tile of 128 rows x 64 tokens its warps' 525 instructions each take some 2000 cycles beside decoding and waits, where the
// special-function unit alone would need 512 and the products 640 (960 with rests): 16384 tokens for 512 rows of 8 heads of 128, 35 GFLOP, 64 us in
// pairs of blocks without rests (550 TFLOP/s, the tensor pipe busy for 27 %), some 88 with.  Few rows or tokens: the chain of four kernels, some 24 us.
// Registers: the softmax's forms with two slots spill, those of weights as two numbers some 240 bytes a thread, the others 40 to 90; a stack frame of 256 bytes
// holds the scores that moved_row looks at.
// Measured and not kept (that case with queries of one number, all kernels, us, of 114 when tried): eight warps of softmax a slot 147; 16 scores at a time in a loop 146; fragments of four
// rows a thread, whose norms then serve four scores 148; both slots in step 122.
//
// Waits are bounded: after the cache's limit (some two seconds unless lq_cache_wait says less) a waiting thread sets LQ_CACHE_GAVE_UP, and all leave, once
// the matrix unit has done what it was given.
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
constexpr float kRoom = 65536.0f, kMostWeight = 16384.0f, kLeastWeight = 4.0f;
constexpr int kLift = 6;
constexpr int kColumns = 512;           // of tensor memory: all (one CTA an SM)

// Shared memory, by address.  Below the table: pieces (a tile's keys or values), then what is small; behind it: the queries, then pieces.
template <int P, bool kTwo, int kRests>
struct Layout {
    static constexpr int kSlots = cache_shared_slots(P, kTwo, kRests), kPanels = P / 64, kPiece = P * 128;
    static constexpr int kBlocks = cache_shared_pairs(P, kTwo, kRests) ? 2 : 1;         // of rows
    // tiles of keys and of values at a time: as many as there is room for
    static constexpr int kKeys = P == 64 ? 3 : P == 256 ? 1 : kBlocks == 2 ? 2 : 3, kValues = P == 64 ? 4 : P == 256 ? 1 : kBlocks == 2 ? 3 : 4;
    static constexpr int kSoftmaxWarps = 4;                             // of a slot: a thread has a row
    static constexpr int kThreads = 32 * kSoftmaxWarps * kSlots + kDecode + 128;
    static constexpr int kDecodeAt = kSoftmaxWarps * kSlots, kIssuer = kDecodeAt + kDecodeWarps;        // warps
    // Registers a thread at launch, and as they are dealt out to softmax, decoding and products: no more than all threads had.
    static constexpr int kRegisters = kSlots == 2 ? 96 : 128, kSoftmax = kSlots == 2 ? 144 : 208, kDecoding = kSlots == 2 ? 72 : 120, kProducts = 40;
    static_assert(32 * kSoftmaxWarps * kSlots * kSoftmax + kDecode * kDecoding + 128 * kProducts <= kThreads * kRegisters && kThreads * kRegisters <= 65536, "registers");
    static constexpr int kQueries = kBlocks * kPanels * kPanelQ;
    static constexpr int kLowPieces = P == 64 ? 7 : P == 128 ? 3 : 1;
    static constexpr int kSmallAt = kSystemBytes + kLowPieces * kPiece;
    static constexpr int kEnd = kHighAt + kQueries + (kKeys + kValues - kLowPieces) * kPiece;
    static __device__ __forceinline__ uint32_t piece(int i) { return i < kLowPieces ? kSystemBytes + i * kPiece : kHighAt + kQueries + (i - kLowPieces) * kPiece; }
    static __device__ __forceinline__ uint32_t keys(int stage) { return piece(stage); }
    static __device__ __forceinline__ uint32_t values(int stage) { return piece(kKeys + stage); }
    static __device__ __forceinline__ uint32_t queries(int slot, int panel) { return kHighAt + (slot * kPanels + panel) * kPanelQ; }
    // tensor memory, columns of a slot: scores, weights (and what their rounding left), sums, what the queries' rounding left
    static constexpr bool kInPlace = kRests == kRestsInPlace;           // weights stand in the scores' place: a slot's next scores wait for its sums
    static constexpr int kScores = 0, kWeights = kInPlace ? kScores : kTile, kSums = kInPlace ? kTile : kTile + (kTwo ? kTile : kTile / 2), kOwnColumns = kSums + P;
    static constexpr bool kShared = kRests && kSlots == 2 && !cache_shared_pairs(P, kTwo, kRests);      // both slots have the same rows, and one copy of their rests
    static constexpr int kSlotColumns = kOwnColumns + (kRests && !kShared ? P / 2 : 0), kAllColumns = kSlots * kSlotColumns + (kShared ? P / 2 : 0);
    static __device__ __forceinline__ uint32_t rests(int slot) { return kShared ? kSlots * kSlotColumns : slot * kSlotColumns + kOwnColumns; }
    static_assert(kAllColumns <= kColumns && kEnd <= 227 << 10, "places");
};

struct Small {
    uint64_t key_full[4], key_empty[4], value_full[4], value_empty[4];  // a place holds a tile's keys or values; they have been read
    uint64_t scored[2], taken[2], weighed[2], summed[2];        // of a slot: its scores are there; have been taken; its weights are there, its sums
    uint64_t brought, rested[2];        // the queries are there; what their rounding left is, of a slot.  (Once each: a wait for a first phase would miss it behind the second.)
    uint64_t drained[4];
    uint32_t tensor;                    // address of tensor memory
    uint32_t failed;
    long long wait_cycles;              // how long a wait may take
    uint32_t seen[4][2];                // of a tile, beside its values: bit per token
    int32_t exponent[4];                // what the values' norms are divided by
    alignas(16) float keys[4][kTile];   // norms
    alignas(16) float values[4][kTile];
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
__device__ __forceinline__ bool gave_up(const Small& sm) { return *reinterpret_cast<const volatile uint32_t*>(&sm.failed); }
// False after the cache's limit, or once another thread has given up.
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, Small& sm, uint32_t* flags)
{
    if (passed(b, parity)) return true;
    const long long start = clock64();
    while (!passed(b, parity)) {
        if (gave_up(sm)) return false;
        if (clock64() - start > sm.wait_cycles) {
            *reinterpret_cast<volatile uint32_t*>(&sm.failed) = 1;
            atomicOr(flags, LQ_CACHE_GAVE_UP);
            return false;
        }
    }
    return true;
}

// Two of them, looked at together.
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity, uint64_t* c, uint32_t other, Small& sm, uint32_t* flags)
{
    const bool x = passed(b, parity), y = passed(c, other);
    return (x || wait(b, parity, sm, flags)) && (y || wait(c, other, sm, flags));
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* b)
{
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" :: "r"(address_of(b)) : "memory");
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
__device__ __forceinline__ void tensor_load16(uint32_t (&v)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_store16(uint32_t at, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// 32 columns of 16 lanes, by 8: registers 4 j and 4 j + 1 of lane l hold columns 8 j + 2 (l % 4) and the next of lane l / 4, the two behind those of lane l / 4 + 8.
__device__ __forceinline__ void tensor_load_rows(uint32_t (&v)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
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

// The products and their commits are given by a whole warp, whose elected lane (always the same one) issues them: what they are given is then the
// same in all lanes.
template <int kRegisters>
__device__ __forceinline__ void give_up_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kRegisters)); }
template <int kRegisters>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kRegisters)); }

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
    asm volatile("{\n\t.reg .pred p, q;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(sums), "l"(a), "l"(b), "r"(how), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void multiply_tensor(uint32_t sums, uint32_t a, uint64_t b, uint32_t how, bool add)
{
    asm volatile("{\n\t.reg .pred p, q;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
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

// ---- the queries -----------------------------------------------------------------------------------------------

// Row i of a head's block b is query r % group of sequence r / group, r = 128 b + i.  The queries go to the workspace first, once for all CTAs that
// take them: turned, times a power of two, as fp16 in the place that the matrix unit expects (panels of 64 coordinates, swizzled), what that
// rounding left in rows, and the factors.  (Each CTA for itself: 300 instructions a row, 18 us for two blocks.)  Rows without a query are zeros.
template <int P>
__device__ __forceinline__ char* block_at(const CacheSharedArgs& a, int head, int block)
{
    const int64_t blocks = ((int64_t)a.batch * a.group + kRows - 1) / kRows;
    return a.rows + (head * blocks + block) * cache_shared_block_bytes(P);
}

// Where chunk `chunk` of 16 bytes of row r stands in a panel of rows of 128 bytes.
__device__ __forceinline__ uint32_t swizzled(int r, int chunk) { return (uint32_t)(r * 128 + ((chunk ^ (r & 7)) << 4)); }

constexpr int kRowWarps = 8;

template <int P, bool kFloat>
__global__ void __launch_bounds__(32 * kRowWarps) shared_rows_kernel(const __grid_constant__ CacheSharedArgs a)
{
    constexpr int kEach = P / 32;                               // coordinates of a lane, side by side
    pdl_wait();
    pdl_launch_next();
    const int lane = threadIdx.x & 31, d0 = lane * kEach, all = a.batch * a.group, padded = (all + kRows - 1) / kRows * kRows;      // (at most 2^26)
    const int64_t item = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    const int head = (int)(item / padded), row = (int)(item - (int64_t)head * padded);
    if (head >= a.shape.heads) return;
    const bool live = row < all;
    const int sequence = live ? row / a.group : 0, query = live ? row - sequence * a.group : 0;
    const CacheRotary& r = a.rotary;
    const int half = r.dim / 2;
    const float* angles = r.table;
    bool lost = false;
    if (r.table && live) {
        int64_t at;
        if (r.at) {
            at = r.at[sequence];
        } else {
            const int64_t before = min((int64_t)max(*a.prefix_length, 0), a.prefix_most), own = min((int64_t)max(a.lengths[sequence], 0), a.own_most);
            at = max(before + own - 1, (int64_t)0);
        }
        lost = at < 0 || at >= r.positions;
        if (lost) { if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION); }
        else angles += at * r.dim;
    }
    const char* const from = static_cast<const char*>(a.queries.data) + (int64_t)sequence * a.queries.token_bytes + (int64_t)(head * a.group + query) * a.queries.head_bytes;
    using Raw = std::conditional_t<kFloat, float, unsigned short>;      // (what its bits mean is looked at when all loads are under way)
    Raw x[kEach], u[kEach];
    float c[kEach], t[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int d = d0 + e;
        const bool there = live && d < a.shape.dim, turned = there && r.table && !lost && d < r.dim;
        const int other = r.interleaved ? d ^ 1 : d < half ? d + half : d - half, p = r.interleaved ? d >> 1 : d < half ? d : d - half;
        x[e] = there ? reinterpret_cast<const Raw*>(from)[d] : (Raw)0;
        u[e] = turned ? reinterpret_cast<const Raw*>(from)[other] : (Raw)0;
        c[e] = turned ? angles[p] : 1.0f;
        t[e] = turned ? angles[half + p] : 0.0f;
    }
    auto number = [&](Raw v) -> float {
        if constexpr (kFloat) return v;
        else return a.queries.type == LQ_BF16 ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
    };
    float y[kEach];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int d = d0 + e;
        y[e] = number(x[e]);
        if (live && r.table && !lost && d < min(r.dim, a.shape.dim)) {
            const bool lower = r.interleaved ? d % 2 == 0 : d < half;
            const float z = number(u[e]);
            y[e] = lower ? __fsub_rn(__fmul_rn(y[e], c[e]), __fmul_rn(z, t[e])) : __fadd_rn(__fmul_rn(y[e], c[e]), __fmul_rn(z, t[e]));
        }
        if (lost) y[e] = __uint_as_float(0x7fffffffu);
        top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    // 2^e brings the largest coordinate to [2^14, 2^15); Inf and NaN stay what they are
    const int up = min(top >= 0x7f800000u || top == 0 ? 0 : 141 - (int)(top >> 23), 120);
    uint32_t h[kEach / 2], rest[kEach / 2];
#pragma unroll
    for (int e = 0; e < kEach; e += 2) {
        const float z = y[e] * power(up), w = y[e + 1] * power(up);
        h[e / 2] = halves(z, w);
        rest[e / 2] = rest_of(h[e / 2], z, w);
    }
    char* const to = block_at<P>(a, head, row / kRows);
    const int place = row % kRows;
    auto store = [&](char* at, const uint32_t (&v)[kEach / 2]) {
        if constexpr (kEach == 2) *reinterpret_cast<uint32_t*>(at) = v[0];
        else if constexpr (kEach == 4) *reinterpret_cast<uint2*>(at) = make_uint2(v[0], v[1]);
        else *reinterpret_cast<uint4*>(at) = make_uint4(v[0], v[1], v[2], v[3]);
    };
    store(to + (d0 >> 6) * kPanelQ + swizzled(place, (d0 & 63) >> 3) + (d0 & 7) * 2, h);
    store(to + 2 * P * kRows + place * 2 * P + d0 * 2, rest);
    if (lane == 0) reinterpret_cast<float*>(to + 4 * P * kRows)[place] = a.scale * power(-up);
}

// ---- a CTA's share ---------------------------------------------------------------------------------------------

struct Share {
    int head, block;                    // of the cache; first block of rows
    int tile0, tiles;                   // its tiles of the prefix
    int64_t length;                     // of the prefix
    bool pair;                          // two blocks of rows; else (two slots) even and odd tiles
};

// The pair of blocks that this CTA takes, and whether it is one.
template <int kSlots, bool kPairs>
__device__ __forceinline__ bool pair_of_blocks(const CacheSharedArgs& a, int* head = nullptr, int* block = nullptr)
{
    constexpr int kAtOnce = kPairs ? kSlots : 1;
    const int blocks = (a.batch * a.group + kRows - 1) / kRows, pairs = (blocks + kAtOnce - 1) / kAtOnce;
    const int item = blockIdx.x / a.splits, h = item / pairs, b = (item - h * pairs) * kAtOnce;
    if (head) { *head = h; *block = b; }
    return kAtOnce == 2 && b + 1 < blocks;
}

template <int kSlots, bool kPairs>
__device__ __forceinline__ Share share_of(const CacheSharedArgs& a)
{
    Share s;
    s.pair = pair_of_blocks<kSlots, kPairs>(a, &s.head, &s.block);
    const int split = blockIdx.x % a.splits;
    const int given = *a.prefix_length;
    s.length = given < 0 ? 0 : given > a.prefix_most ? a.prefix_most : given;
    const int64_t all = (s.length + kTile - 1) / kTile;
    s.tile0 = (int)(all * split / a.splits);
    s.tiles = (int)(all * (split + 1) / a.splits) - s.tile0;
    return s;
}

// ---- decoding --------------------------------------------------------------------------------------------------

// A thread decodes 64 coordinates of a token at a time, a row of 128 bytes of a panel: lanes have tokens in a row, so that their stores, swizzled, meet
// every bank.  A warp's are all keys or all values.
template <int P>
struct Codes {
    static constexpr int kItems = 2 * (P / 64) * (kTile / 32);          // of 32 tokens
    static constexpr int kEach = (kItems + kDecodeWarps - 1) / kDecodeWarps;
    static constexpr int kNorms = (kItems - 1) % kDecodeWarps;          // the warp that brings the norms: one that has values
    uint32_t w[kEach][16];              // (symbols of 4 bits: 8 words)
    float keys[2], values[2];           // norms, brought by one warp
    uint32_t seen;                      // bit i: the tile's i-th 16 tokens are on a page that is there
};

template <int P>
__device__ __forceinline__ void item_of(int i, int& kind, int& panel, int& token)
{
    kind = i / (Codes<P>::kItems / 2);
    panel = i / (kTile / 32) % (P / 64);
    token = i % (kTile / 32) * 32;
}

// The page of 16 of a tile's tokens, by lanes 0 to 3, as the table has it (no look is taken at it before it is used).
__device__ __forceinline__ int page_of(const CacheSharedArgs& a, const Share& s, int tile, bool inside, int lane)
{
    const int64_t token = (int64_t)(s.tile0 + tile) * kTile + 16 * lane;
    return inside && lane < kTile / 16 && token < s.length ? a.prefix[token >> a.shape.page_shift] : -1;
}

__device__ __forceinline__ void load32(uint32_t* v, const char* from)
{
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "l"(from) : "memory");
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(from + 16) : "memory");
}

// Where there is no page, the level tables are read instead (any numbers will do: the token is not seen): nothing then waits for a load here.
template <int P>
__device__ __forceinline__ void fetch(Codes<P>& c, const CacheSharedArgs& a, const Share& s, int tile, int page, int warp, int lane)
{
    const int mask = (1 << a.shape.page_shift) - 1;
    const int row0 = (s.tile0 + tile) * kTile & mask;
    const bool there = (uint32_t)page < (uint32_t)a.num_pages;
    c.seen = __ballot_sync(0xffffffffu, there) & 15u;
    if (c.seen != 15u && lane < kTile / 16 && !there && (int64_t)(s.tile0 + tile) * kTile + 16 * lane < s.length) atomicOr(a.flags, LQ_CACHE_BAD_PAGE);
    const uint32_t values_at = (uint32_t)a.shape.row_words[0] << a.shape.page_shift, norms_at = values_at + ((uint32_t)a.shape.row_words[1] << a.shape.page_shift);
    const char* const pages = reinterpret_cast<const char*>(a.pages + (int64_t)s.head * a.shape.head_words);
    const uint32_t page_bytes = 4u * (uint32_t)a.shape.page_words;
#pragma unroll
    for (int k = 0; k < Codes<P>::kEach; ++k) {
        const int i = warp + kDecodeWarps * k;
        if (i >= Codes<P>::kItems) break;
        int kind, panel, token;
        item_of<P>(i, kind, panel, token);
        token += lane;
        const int p = __shfl_sync(0xffffffffu, page, token >> 4), bits = kind ? a.shape.sym_bits[1] : a.shape.sym_bits[0];
        const uint32_t words = kind ? a.shape.row_words[1] : a.shape.row_words[0];
        const uint32_t at = 4u * ((kind ? values_at : 0u) + (uint32_t)((row0 + token) & mask) * words) + (uint32_t)(panel * 8 * bits);
        const char* from = pages + (uint64_t)(uint32_t)p * page_bytes + at;
        from = (uint32_t)p < (uint32_t)a.num_pages ? from : reinterpret_cast<const char*>(a.tables);
        load32(c.w[k], from);
        if (bits == 8) load32(c.w[k] + 8, from + 32);
    }
    if (warp == Codes<P>::kNorms) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int token = lane + 32 * i, p = __shfl_sync(0xffffffffu, page, token >> 4);
            const float* norms = reinterpret_cast<const float*>(pages + (uint64_t)(uint32_t)p * page_bytes) + norms_at + ((row0 + token) & mask);
            norms = (uint32_t)p < (uint32_t)a.num_pages ? norms : a.tables->levels;
            c.keys[i] = norms[0];
            c.values[i] = norms[(uint32_t)p < (uint32_t)a.num_pages ? mask + 1 : 0];
        }
    }
}

// A warp's k-th item into its piece.
template <int P>
__device__ __forceinline__ void decode(const Codes<P>& c, int k, const CacheSharedArgs& a, uint32_t piece, int warp, int lane)
{
    int kind, panel, token;
    item_of<P>(warp + kDecodeWarps * k, kind, panel, token);
    token += lane;
    const uint32_t row = piece + panel * kPanel + token * 128, copies = kTableAt + 4 * lane + 128 * kind;
    const uint32_t turn = (token & 7) << 4;
    const uint32_t (&w)[16] = c.w[k];
    // (16 look-ups before their stores: the compiler moves no load of shared memory above a store)
    if ((kind ? a.shape.sym_bits[1] : a.shape.sym_bits[0]) == 8) {
        auto two = [](uint32_t x, uint32_t y) { return __byte_perm(x, y, 0x5410); };
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            uint32_t v[8];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const uint32_t x = w[2 * j + m];
                v[2 * m] = two(look<0>(x, copies), look<1>(x, copies));
                v[2 * m + 1] = two(look<2>(x, copies), look<3>(x, copies));
            }
            store16(row + ((16 * j) ^ turn), v[0], v[1], v[2], v[3]);
            store16(row + ((16 * j + 16) ^ turn), v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
            uint32_t v[4][4];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                v[m][0] = look<0>(w[j + m], copies); v[m][1] = look<1>(w[j + m], copies);
                v[m][2] = look<2>(w[j + m], copies); v[m][3] = look<3>(w[j + m], copies);
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) store16(row + ((16 * (j + m)) ^ turn), v[m][0], v[m][1], v[m][2], v[m][3]);
        }
    }
}

// ... and the norms beside its values, by one warp.
template <int P>
__device__ __forceinline__ void place_norms(const Codes<P>& c, const Share& s, Small& sm, int tile, int stage, int lane)
{
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

// A weight's factor 2^up is at most 2^kFar.  It is part of p's exponent, so that p below 2^(-126 - up) would be lost to the denominator: no less than 2^-kLeast,
// where p (at most 2^16) times a norm (below 2) is 0 as fp16 already, as it is for every lesser factor.  Terms down to 2^-82 of the reference's then count.
constexpr int kFar = 100, kLeast = 44;
static_assert(16 + 1 - kLeast < -25, "such a weight rounds to 0");

// Reference and scale of a warp's rows as a tile of scores `v` wants them, the denominators and the sums (`summed`: a barrier's phase that they wait for; NULL:
// there are none yet) moved along.  Both numbers are whole, so that what has been summed is multiplied by powers of two.  (Not inline: it is
// rare, and what it wants to keep in registers crowds out what the usual way needs.)
template <int P>
__device__ __noinline__ Row moved_row(Row row, Small& sm, const uint32_t* v, int stage, uint64_t* summed, uint32_t parity, uint32_t sums, uint32_t* flags)
{
    const float* const keys = sm.keys[stage];
    const uint32_t seen[2] = {sm.seen[stage][0], sm.seen[stage][1]};
    float most = -INFINITY;
    bool none_such = false;         // a score that is not a number: nothing is gained by waiting for a better one
#pragma unroll 8
    for (int j = 0; j < kTile; ++j) {
        const float d = seen[j / 32] >> (j % 32) & 1 ? fmaf(__uint_as_float(v[j]) * row.f, keys[j], -row.ref) : -INFINITY;
        most = fmaxf(most, d);
        none_such = none_such || d != d;
    }
    const float step = ceilf(row.begun ? fmaxf(most, 0.0f) : most);
    float moved = 0.0f;
    if (step > -INFINITY) {
        const float ref = row.ref + step;
        moved = row.ref - ref;
        row.ref = ref;
        if (row.begun) row.total *= ex2(moved);
    }
    float heavy = 0.0f;
#pragma unroll 8
    for (int j = 0; j < kTile; ++j)
        if (seen[j / 32] >> (j % 32) & 1) heavy = fmaxf(heavy, ex2(fmaf(__uint_as_float(v[j]) * row.f, keys[j], -row.ref)) * sm.values[stage][j]);
    // the largest weight is 2^(exponent + e) or up to twice that
    const int exponent = sm.exponent[stage], e = exponent_of(heavy), by = (int)fmaxf(moved, -4000.0f);
    int scale = max(exponent + e, exponent + kLift - kFar + 6);
    if (row.begun) scale = max(scale, max(row.scale + by, -4000));
    const int down = row.begun ? by + row.scale - scale : -4000;   // (at most 0)
    const float factor = down < -126 ? 0.0f : power(down);
    row.scale = scale;
    row.begun = row.begun || most > -INFINITY || none_such;
    if (summed) {
        wait(summed, parity, sm, flags);        // (a failure is met by the next wait, too)
        __syncwarp();
        fence_after();
#pragma unroll 1
        for (int c = 0; c < P; c += 16) {
            uint32_t x[16];
            tensor_load16(x, sums + c);
            loaded();
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * factor);
            tensor_store16(sums + c, x);
        }
        stored();
    }
    return row;
}

// The softmax of a slot's uses.  A row's scores become weights in one pass with reference and scale as they are, and once more if that shows that these have to
// move (p is fp32 and has room: a tile's may add up to kRoom; a weight is fp16, up to kMostWeight).  The scale of the weights is part of p's exponent,
// and taken out of the denominator again.
template <int P, bool kTwo, int kRests>
struct Softmax {
    using L = Layout<P, kTwo, kRests>;
    Row row;
    int slot;
    uint32_t columns;                   // of tensor memory, this slot's

    // A row's first tile: the reference is its largest score, the scale that of a weight of 1 at the tile's largest norm (if that is far too high,
    // the pass shows it).
    __device__ __forceinline__ void begin(Small& sm, int stage)
    {
        float most = -INFINITY;
        bool none_such = false;         // a score that is not a number: nothing is gained by waiting for a better one
#pragma unroll 1
        for (int c = 0; c < kTile; c += 16) {
            uint32_t x[16];
            tensor_load16(x, columns + L::kScores + c);
            loaded();
            const uint32_t seen = sm.seen[stage][c / 32] >> (c % 32);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float d = seen >> j & 1 ? __uint_as_float(x[j]) * row.f * sm.keys[stage][c + j] : -INFINITY;
                most = fmaxf(most, d);
                none_such = none_such || d != d;
            }
        }
        if (row.begun) return;
        if (most > -INFINITY) row.ref = ceilf(most);
        row.scale = sm.exponent[stage];
        row.begun = most > -INFINITY || none_such;
    }

    // The n-th tile of this slot, whose norms are at `stage`.
    __device__ __forceinline__ void tile(Small& sm, int stage, int n, uint32_t* flags)
    {
        const int exponent = sm.exponent[stage];
        const uint32_t seen[2] = {sm.seen[stage][0], sm.seen[stage][1]};
        const bool fresh = !row.begun;
        if (__any_sync(0xffffffffu, fresh)) begin(sm, stage);
        uint32_t v[kTile], w[kTile / 2], rest[kTwo ? kTile / 2 : 1];
        tensor_load32(reinterpret_cast<uint32_t (&)[32]>(v[0]), columns + L::kScores);
        tensor_load32(reinterpret_cast<uint32_t (&)[32]>(v[32]), columns + L::kScores + 32);
        loaded();
        fence_before();
        arrive(&sm.taken[slot]);        // (the next tile's scores may come)
        float sum;
#pragma unroll 1
        for (int tries = 0;; ++tries) {
            const int wanted = exponent - row.scale + kLift, up = max(-kLeast, min(kFar, wanted));
            const float offset = (float)up - row.ref;
            const uint64_t f2 = pair_of(row.f, row.f), offset2 = pair_of(offset, offset);
            uint64_t total[2] = {0, 0};
            __half2 heavy = __half2half2(__ushort_as_half(0));
            auto pass = [&](auto all) {
#pragma unroll
                for (int j = 0; j < kTile; j += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(&sm.keys[stage][j]), m = *reinterpret_cast<const float4*>(&sm.values[stage][j]);
                    float x, y, z, u;
                    parted(fma2(mul2(pair_of(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), f2), pair_of(k.x, k.y), offset2), x, y);
                    parted(fma2(mul2(pair_of(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])), f2), pair_of(k.z, k.w), offset2), z, u);
                    if constexpr (!decltype(all)::value) {
                        const uint32_t bits = seen[j / 32] >> (j % 32);
                        x = bits & 1 ? x : -INFINITY; y = bits & 2 ? y : -INFINITY; z = bits & 4 ? z : -INFINITY; u = bits & 8 ? u : -INFINITY;
                    }
                    const uint64_t p = pair_of(ex2(x), ex2(y)), q = pair_of(ex2(z), ex2(u));
                    total[0] = add2(total[0], p);
                    total[1] = add2(total[1], q);
                    parted(mul2(p, pair_of(m.x, m.y)), x, y);
                    parted(mul2(q, pair_of(m.z, m.w)), z, u);
                    w[j / 2] = halves(x, y);
                    w[j / 2 + 1] = halves(z, u);
                    if constexpr (kTwo) { rest[j / 2] = rest_of(w[j / 2], x, y); rest[j / 2 + 1] = rest_of(w[j / 2 + 1], z, u); }
                    heavy = __hmax2(heavy, __hmax2(reinterpret_cast<const __half2&>(w[j / 2]), reinterpret_cast<const __half2&>(w[j / 2 + 1])));
                }
            };
            if ((seen[0] & seen[1]) == 0xffffffffu) pass(std::true_type()); else pass(std::false_type());
            float x, y;
            parted(add2(total[0], total[1]), x, y);
            sum = (x + y) * power(-up);
            const float largest = __half2float(__hmax(__low2half(heavy), __high2half(heavy)));
            const bool over = sum > kRoom || largest >= kMostWeight || wanted > kFar || (fresh && row.begun && largest < kLeastWeight);
            if (tries > 0 || !__any_sync(0xffffffffu, over)) break;
            if (fresh) row.begun = false;
            uint32_t kept[kTile];
#pragma unroll
            for (int j = 0; j < kTile; ++j) kept[j] = v[j];
            row = moved_row<P>(row, sm, kept, stage, n > 0 ? &sm.summed[slot] : nullptr, (n - 1) & 1, columns + L::kSums, flags);
        }
        row.total += sum;
        if (n > 0) {                    // the weights before have been used
            wait(&sm.summed[slot], (n - 1) & 1, sm, flags);
            __syncwarp();
            fence_after();
        }
        tensor_store32(columns + L::kWeights, w);
        if constexpr (kTwo) tensor_store32(columns + L::kWeights + 32, rest);
        stored();
    }
};

// ---- products ------------------------------------------------------------------------------------------------

// Scores of a slot's uses, by one warp, and weighted values by another: each waits only for what its own products need.
template <int P, bool kTwo, int kRests>
__device__ __forceinline__ void issue_scores(const CacheSharedArgs& a, const Share& s, Small& sm, uint32_t tensor, int slot)
{
    using L = Layout<P, kTwo, kRests>;
    constexpr uint32_t how = instruction(kTile, false);
    const uint32_t at = tensor + slot * L::kSlotColumns;
    bool ok = wait(&sm.brought, 0, sm, a.flags);
    if constexpr (kRests)               // (what the queries' rounding left is there)
        for (int w = L::kShared ? 0 : slot; w < (L::kShared ? L::kSlots : slot + 1); ++w) ok = wait(&sm.rested[w], 0, sm, a.flags) && ok;
    const uint64_t queries = operand(L::queries(s.pair ? slot : 0, 0), 16);
    for (int tile = s.pair ? 0 : slot, n = 0; tile < s.tiles; tile += s.pair ? 1 : L::kSlots, ++n) {
        const int stage = tile % L::kKeys;
        ok = wait(&sm.key_full[stage], (tile / L::kKeys) & 1, L::kInPlace ? &sm.summed[slot] : &sm.taken[slot], (n - 1) & 1, sm, a.flags) && ok;         // (there is no phase before the first to wait for)
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        fence_after();
        const uint64_t keys = operand(L::keys(stage), 16);
        // (the rests first: each step cuts the sum's last bit off, which is worth nothing while the sum is small)
        if constexpr (kRests)
#pragma unroll
            for (int k = 0; k < P / 16; ++k)
                multiply_tensor(at + L::kScores, tensor + L::rests(slot) + 8 * k, keys + (k / 4 * kPanel + k % 4 * 32 >> 4), how, k > 0);
#pragma unroll
        for (int k = 0; k < P / 16; ++k)
            multiply(at + L::kScores, queries + (k / 4 * kPanelQ + k % 4 * 32 >> 4), keys + (k / 4 * kPanel + k % 4 * 32 >> 4), how, kRests != 0 || k > 0);
        commit(&sm.scored[slot]);
        commit(&sm.key_empty[stage]);
    }
}

template <int P, bool kTwo, int kRests>
__device__ __forceinline__ void issue_sums(const CacheSharedArgs& a, const Share& s, Small& sm, uint32_t tensor, int slot)
{
    using L = Layout<P, kTwo, kRests>;
    constexpr uint32_t how = instruction(P, true);
    const uint32_t at = tensor + slot * L::kSlotColumns;
    bool ok = true;
    for (int tile = s.pair ? 0 : slot, n = 0; tile < s.tiles; tile += s.pair ? 1 : L::kSlots, ++n) {
        const int stage = tile % L::kValues;
        ok = wait(&sm.value_full[stage], (tile / L::kValues) & 1, &sm.weighed[slot], n & 1, sm, a.flags) && ok;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        fence_after();
        const uint64_t values = operand(L::values(stage), kPanel);
#pragma unroll
        for (int rest = 0; rest < (kTwo ? 2 : 1); ++rest)
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
                multiply_tensor(at + L::kSums, at + L::kWeights + 32 * rest + 8 * k, values + k * (2048 >> 4), how, n > 0 || rest > 0 || k > 0);
        commit(&sm.summed[slot]);
        commit(&sm.value_empty[stage]);
    }
}

// ---- the kernel ------------------------------------------------------------------------------------------------

template <int P, bool kTwo, int kRests>
__global__ void __launch_bounds__(Layout<P, kTwo, kRests>::kThreads, 1) shared_prefix_kernel(const __grid_constant__ CacheSharedArgs a)
{
    using L = Layout<P, kTwo, kRests>;
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
            constexpr int kItems = Codes<P>::kItems / 2;                // warps that bring a tile's keys, or values
            const int readers = pair_of_blocks<L::kSlots, cache_shared_pairs(P, kTwo, kRests)>(a) ? 2 : 1;   // slots that read them
            for (int i = 0; i < 4; ++i) {
                barrier_init(&sm.key_full[i], 32 * kItems); barrier_init(&sm.key_empty[i], readers);
                barrier_init(&sm.value_full[i], 32 * kItems); barrier_init(&sm.value_empty[i], readers);
            }
            for (int i = 0; i < 2; ++i) {
                barrier_init(&sm.scored[i], 1); barrier_init(&sm.taken[i], 32 * L::kSoftmaxWarps);
                barrier_init(&sm.weighed[i], 32 * L::kSoftmaxWarps); barrier_init(&sm.summed[i], 1);
                barrier_init(&sm.rested[i], 32 * L::kSoftmaxWarps);
            }
            barrier_init(&sm.brought, 1);
            for (int i = 0; i < 4; ++i) barrier_init(&sm.drained[i], 1);
            sm.failed = a.wait_cycles == 0;     // (nothing is brought then)
            sm.wait_cycles = a.wait_cycles;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(address_of(&sm.tensor)), "n"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    pdl_wait();
    pdl_launch_next();
    const Share s = share_of<L::kSlots, cache_shared_pairs(P, kTwo, kRests)>(a);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tensor = sm.tensor;
    // slot s of a use: pairs of blocks take every tile twice
    constexpr int slots = L::kSlots;
    const int uses = s.pair ? 2 * s.tiles : s.tiles;
    auto tile_of = [&](int use) { return s.pair ? use >> 1 : use; };

    const int slot = warp / L::kSoftmaxWarps, place = tid & 127;        // of the softmax's warps: the slot; the thread's row of the block
    const int64_t my_row = (int64_t)(s.block + (s.pair ? slot : 0)) * kRows + place;
    const uint32_t lanes = tensor + ((uint32_t)(32 * (warp & 3)) << 16), mine = lanes + slot * L::kSlotColumns;
    if (warp < L::kDecodeAt) {
        // ---- softmax: a thread has a row
        take_registers<L::kSoftmax>();
        const char* const queries = block_at<P>(a, s.head, s.block + (s.pair ? slot : 0));
        Softmax<P, kTwo, kRests> softmax;
        softmax.slot = slot; softmax.columns = mine;
        Row& row = softmax.row;
        row.f = reinterpret_cast<const float*>(queries + 4 * P * kRows)[place];
        if constexpr (kRests) {                                         // what the queries' rounding left goes to tensor memory
            const uint4* from = reinterpret_cast<const uint4*>(queries + 2 * P * kRows + place * 2 * P);
#pragma unroll 1
            for (int p = L::kShared ? slot : 0; p < L::kPanels; p += L::kShared ? L::kSlots : 1) {
                uint32_t v[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 x = from[8 * p + i];
                    v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
                }
                tensor_store32(lanes + L::rests(slot) + 32 * p, v);
            }
            stored();
            fence_before();
            arrive(&sm.rested[slot]);
        }
        const bool live = __any_sync(0xffffffffu, my_row < (int64_t)a.batch * a.group);
        int n = 0;
        bool ok = true;
        for (int use = slot; use < uses && ok; use += slots, ++n) {
            const int tile = tile_of(use), stage = tile % L::kValues;
            ok = wait(&sm.value_full[stage], (tile / L::kValues) & 1, &sm.scored[slot], n & 1, sm, a.flags);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            fence_after();
            if (live) softmax.tile(sm, stage, n, a.flags);
            else {                      // (its arrivals must not run ahead of the others' by a tile)
                arrive(&sm.taken[slot]);
                if (n > 0) wait(&sm.summed[slot], (n - 1) & 1, sm, a.flags);
            }
            fence_before();
            arrive(&sm.weighed[slot]);
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, wait(&sm.summed[slot], (n - 1) & 1, sm, a.flags));
        fence_after();
        if (live) {
            // ---- what is left of this row; of a block that is alone, one part of even tiles and one of odd ones
            const int part = blockIdx.x % a.splits + (slot == 1 && !s.pair ? a.splits : 0);
            const int64_t all_rows = (int64_t)a.batch * a.shape.heads * a.group;
            const int all = a.batch * a.group;
            auto part_of = [&](int r) {
                const int sequence = r / a.group;
                return a.parts + (part * all_rows + (int64_t)sequence * a.shape.heads * a.group + s.head * a.group + (r - sequence * a.group)) * cache_part_floats(P);
            };
            if (n > 0 && ok) {
                // four lanes have 32 bytes of a row side by side: lane l those of rows l / 4, + 8, + 16 and + 24
                const int row0 = (int)my_row - lane + lane / 4;
                float* to[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = row0 + 8 * i < all ? part_of(row0 + 8 * i) + 2 * (lane & 3) : nullptr;
#pragma unroll 1
                for (int c = 0; c < P; c += 32) {
                    uint32_t v[2][16];
                    tensor_load_rows(v[0], mine + L::kSums + c);
                    tensor_load_rows(v[1], mine + L::kSums + c + (16u << 16));
                    loaded();
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (to[i])
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                *reinterpret_cast<uint2*>(to[i] + c + 8 * j) = make_uint2(v[i / 2][4 * j + 2 * (i & 1)], v[i / 2][4 * j + 2 * (i & 1) + 1]);
                }
            }
            if (my_row < all)
                *reinterpret_cast<float4*>(part_of((int)my_row) + P) = make_float4(row.begun ? row.ref : kLow, (float)(row.scale - kLift), n > 0 && ok ? row.total : 0.0f, 0.0f);
        }
        fence_before();
    } else if (warp < L::kIssuer) {
        // ---- decoding: codes a tile ahead, page numbers three
        give_up_registers<L::kDecoding>();
        const int t = warp - L::kDecodeAt;
        Codes<P> codes;
        const int page = page_of(a, s, 0, s.tiles > 0, lane);
        int next = page_of(a, s, 1, s.tiles > 1, lane), after = page_of(a, s, 2, s.tiles > 2, lane);
        if (s.tiles > 0) fetch<P>(codes, a, s, 0, page, t, lane);
        for (int tile = 0; tile < s.tiles && t < Codes<P>::kItems && !__any_sync(0xffffffffu, gave_up(sm)); ++tile) {
            const Codes<P> now = codes;
            if (tile + 1 < s.tiles) fetch<P>(codes, a, s, tile + 1, next, t, lane);
            next = after;
            after = page_of(a, s, tile + 3, tile + 3 < s.tiles, lane);
            bool ok = true;
#pragma unroll
            for (int k = 0; k < Codes<P>::kEach && ok; ++k) {
                int kind, panel, token;
                item_of<P>(t + kDecodeWarps * k, kind, panel, token);
                const int stage = kind ? tile % L::kValues : tile % L::kKeys, round = kind ? tile / L::kValues : tile / L::kKeys;
                ok = __all_sync(0xffffffffu, wait(kind ? &sm.value_empty[stage] : &sm.key_empty[stage], (round & 1) ^ 1, sm, a.flags));
                if (!ok) break;
                if (kind && t == Codes<P>::kNorms) place_norms<P>(now, s, sm, tile, stage, lane);
                decode<P>(now, k, a, kind ? L::values(stage) : L::keys(stage), t, lane);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                arrive(kind ? &sm.value_full[stage] : &sm.key_full[stage]);
            }
            if (!ok) break;
        }
    } else {
        give_up_registers<L::kProducts>();
        // ---- products: of each slot, a warp for the scores and one for the sums; the first of all brings the queries
        const int me = warp - L::kIssuer, slot_of = me >> 1;
        if (me == 0) {
            const int there = s.pair ? 2 : 1;
            if (lane == 0) {
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(address_of(&sm.brought)), "r"(there * L::kPanels * kPanelQ) : "memory");
                for (int i = 0; i < there; ++i)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 :: "r"(L::queries(i, 0)), "l"(block_at<P>(a, s.head, s.block + i)), "r"(L::kPanels * kPanelQ), "r"(address_of(&sm.brought)) : "memory");
            }
            __syncwarp();
        }
        if (slot_of < L::kSlots) {
            const uint32_t at = __shfl_sync(0xffffffffu, tensor, 0);
            if (me & 1) issue_sums<P, kTwo, kRests>(a, s, sm, at, slot_of);
            else issue_scores<P, kTwo, kRests>(a, s, sm, at, slot_of);
        }
    }
    __syncthreads();
    if (gave_up(sm)) {                  // what is under way ends before tensor memory and shared memory are given back
        const int me = warp - L::kIssuer;
        if (me >= 0 && me < 2 * L::kSlots) {
            commit(&sm.drained[me]);
            const long long start = clock64();
            while (!(passed(&sm.drained[me], 0) && passed(&sm.brought, 0)) && clock64() - start < kCacheMostWait) {}
        }
        if (tid == 0) atomicOr(a.flags, LQ_CACHE_GAVE_UP);
        __syncthreads();
    }
    if (warp == L::kIssuer) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tensor), "n"(kColumns));
    }
}

// ---- the join --------------------------------------------------------------------------------------------------

// What a row's parts of the prefix and of its own tokens give, in an order that goes by their number alone: `share` warps a row, each with some of the parts, of
// which all that has to be read is asked for before anything waits; then their sums in order.
constexpr int kJoinWarps = 8;

template <int P>
__global__ void __launch_bounds__(32 * kJoinWarps) shared_join_kernel(const __grid_constant__ CacheSharedArgs a, int share)
{
    constexpr int kVectors = P / 128 > 0 ? P / 128 : 1;
    __shared__ float4 sums[kJoinWarps][kVectors][32];
    pdl_wait();
    pdl_launch_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp % share;
    const int64_t all_rows = (int64_t)a.batch * a.shape.heads * a.group, row = (int64_t)blockIdx.x * (kJoinWarps / share) + warp / share;
    const bool there = row < all_rows;
    if (blockIdx.x == 0 && threadIdx.x == 0 && (*a.prefix_length < 0 || *a.prefix_length > a.prefix_most)) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
    const int heads = a.shape.heads * a.group, sequence = there ? (int)(row / heads) : 0, head = there ? (int)(row - (int64_t)sequence * heads) : 0;
    const int64_t in_head = (int64_t)sequence * a.group + head % a.group;
    // (where no sequence has a page of its own, no other kernel looks at its length)
    if (there && a.own_most == 0 && head == 0 && mine == 0 && lane == 0 && a.lengths[sequence] != 0) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
    const int blocks = (int)(((int64_t)a.batch * a.group + kRows - 1) / kRows), block = (int)(in_head / kRows);
    const bool alone = a.slots == 2 && (!a.pairs || (blocks % 2 == 1 && block == blocks - 1));
    const int before = a.splits * (alone ? 2 : 1), parts = there ? before + (a.own_most > 0 && a.lengths[sequence] > 0) : 0;
    const float* const prefix = fresh(a.parts);
    const float* const own = fresh(a.own);
    auto part = [&](int i) { return (i < before ? prefix + (i * all_rows + row) * cache_part_floats(P) : own + row * cache_part_floats(P)); };
    auto stats = [&](int i) { return __ldcg(reinterpret_cast<const float4*>(part(i) + P)); };
    // every warp of a row looks at all parts' references, scales and denominators
    float r = kLow, scale = -1000.0f, total = 0.0f;
    for (int i = lane; i < parts; i += 32) {
        const float4 t = stats(i);
        const float r1 = fmaxf(r, t.x), old = r - r1, there = t.x - r1;
        total = total * ex2(old) + t.z * ex2(there);
        scale = fmaxf(scale + old, t.z != 0.0f ? t.y + there : -INFINITY);
        r = r1;
    }
    {
        float most = r;
#pragma unroll
        for (int o = 16; o > 0; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        total *= ex2(r - most);
        scale += r - most;
        r = most;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        scale = fmaxf(scale, __shfl_xor_sync(0xffffffffu, scale, o));
        total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    scale = floorf(fmaxf(scale, -1000.0f));
    float4 acc[kVectors] = {};
    for (int base = mine; base < parts; base += 32 * share) {
        // lane l: the factor of this warp's l-th part from here; 0 where nothing was seen (and nothing written)
        const int i = base + share * lane;
        float f = 0.0f;
        if (i < parts) {
            const float4 t = stats(i);
            if (t.z != 0.0f) f = ex2((t.x - r) + (t.y - scale));
        }
        const int here = min(32, (parts - base + share - 1) / share);
        for (int l = 0; l < here; l += 4) {
            float4 v[4][kVectors];
            float g[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[j] = __shfl_sync(0xffffffffu, f, (l + j) & 31);
                const bool some = l + j < here && g[j] != 0.0f;
                if (!some) g[j] = 0.0f;
#pragma unroll
                for (int k = 0; k < kVectors; ++k)
                    v[j][k] = some && (P >= 128 || lane < P / 4) ? __ldcg(reinterpret_cast<const float4*>(part(base + share * (l + j)) + 4 * (lane + 32 * k)))
                                                                 : make_float4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < kVectors; ++k) {
                    acc[k].x += v[j][k].x * g[j]; acc[k].y += v[j][k].y * g[j]; acc[k].z += v[j][k].z * g[j]; acc[k].w += v[j][k].w * g[j];
                }
        }
    }
    if (share > 1) {
#pragma unroll
        for (int k = 0; k < kVectors; ++k) sums[warp][k][lane] = acc[k];
        __syncthreads();
        if (mine > 0) return;
        for (int w = 1; w < share; ++w)
#pragma unroll
            for (int k = 0; k < kVectors; ++k) {
                const float4 v = sums[warp + w][k][lane];
                acc[k].x += v.x; acc[k].y += v.y; acc[k].z += v.z; acc[k].w += v.w;
            }
    }
    if (!there) return;
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

template <int P, bool kTwo, int kRests>
cudaError_t launch_prefix(const CacheSharedArgs& a, cudaStream_t s)
{
    using L = Layout<P, kTwo, kRests>;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = opt_in_shared_memory(configured, L::kEnd, shared_prefix_kernel<P, kTwo, kRests>);
    // registers are dealt out anew in the kernel: it must have been given as many as that counts on
    static std::atomic<int> registers{0};
    if (e == cudaSuccess && !registers.load(std::memory_order_relaxed)) {
        cudaFuncAttributes at;
        e = cudaFuncGetAttributes(&at, shared_prefix_kernel<P, kTwo, kRests>);
        if (e == cudaSuccess && at.numRegs != L::kRegisters) e = cudaErrorLaunchOutOfResources;
        if (e == cudaSuccess) registers.store(at.numRegs, std::memory_order_relaxed);
    }
    const int64_t blocks = ((int64_t)a.batch * a.group + kRows - 1) / kRows, items = a.shape.heads * (a.pairs ? (blocks + 1) / 2 : blocks);
    if (e == cudaSuccess) e = launch(shared_prefix_kernel<P, kTwo, kRests>, (unsigned)(items * a.splits), L::kThreads, L::kEnd, s, a);
    return e;
}

template <int P>
cudaError_t launch_prefix_of(const CacheSharedArgs& a, cudaStream_t s)
{
    if (a.queries.type != LQ_BF16) return a.rests ? launch_prefix<P, true, kRestsBeside>(a, s) : launch_prefix<P, true, 0>(a, s);
    if constexpr (P == 128) { if (a.rests == kRestsInPlace) return launch_prefix<P, false, kRestsInPlace>(a, s); }
    return a.rests ? launch_prefix<P, false, kRestsBeside>(a, s) : launch_prefix<P, false, 0>(a, s);
}

template <int P>
cudaError_t launch_rows(const CacheSharedArgs& a, cudaStream_t s)
{
    const int64_t rows = ((int64_t)a.batch * a.group + kRows - 1) / kRows * kRows * a.shape.heads;
    const unsigned grid = (unsigned)((rows + kRowWarps - 1) / kRowWarps);
    return a.queries.type == LQ_F32 ? launch(shared_rows_kernel<P, true>, grid, 32 * kRowWarps, 0, s, a) : launch(shared_rows_kernel<P, false>, grid, 32 * kRowWarps, 0, s, a);
}

template <int P>
cudaError_t launch_join(const CacheSharedArgs& a, cudaStream_t s)
{
    const int64_t rows = (int64_t)a.batch * a.shape.heads * a.group;
    // Warps a row: each reads all parts' references and its share of the sums.  Eight, four and two of them, us of the whole call (8 heads, 4 queries each, bf16,
    // prefixes of 512, 8192 and 32768): 256 rows 23.2, 32.3, 55.6 | 23.3, 33.4, 56.8 | 24.1, 35.6, 59.1; 512 rows 26.0, 35.5, 59.3 | 24.4, 34.8, 58.7 | 25.0, 37.0, 61.1;
    // 1152 rows 31.4, 45.2, 84.4 | 27.7, 41.9, 80.9 | 27.2, 41.6, 80.2; 2048 rows 43.0, 58.3, 97.8 | 36.5, 51.6, 90.5 | 35.2, 50.4, 89.6.
    const int share = rows <= 3 * a.sms ? 8 : rows <= 7 * a.sms ? 4 : 2, per = kJoinWarps / share;
    return launch(shared_join_kernel<P>, (unsigned)((rows + per - 1) / per), 32 * kJoinWarps, 0, s, a, share);
}

}  // namespace

int cache_shared_splits(int heads, bool pairs, int64_t rows, int64_t prefix_tokens, int type, int sms)
{
    const int64_t blocks = (rows + kRows - 1) / kRows, items = heads * (pairs ? (blocks + 1) / 2 : blocks), tiles = (prefix_tokens + kTile - 1) / kTile;
    if (tiles == 0) return 0;
    // a tile of two blocks takes twice as long as one of a block alone; what a CTA takes besides is some 8 of those
    const int64_t each = blocks > 1 && pairs ? 2 : 1;
    // The matrix unit cuts off what a sum's last bit does not hold, in every step of 16 tokens (of both numbers of a weight): up to 2^-23 of the sum so far, on
    // average 2^-24 of the last, and all one way.  A sum of fp32 outputs has 1024 tokens at most (2^-17 at worst, 2^-20.7 measured), of fp16 8192 and of bf16
    // 131072: a quarter of half a step of the output at worst.  (Without: 524288 tokens of 148 heads, fp16: a step and a half off.)
    const int64_t most = type == LQ_F32 ? 16 : type == LQ_F16 ? 128 : 2048;
    int64_t best = 1, cost = INT64_MAX;
    for (int64_t n = (tiles + most - 1) / most; n <= tiles; ++n) {
        const int64_t c = (items * n + sms - 1) / sms * ((tiles + n - 1) / n * each + 8);
        if (c < cost) { cost = c; best = n; }
        if (n >= 64 && n * items > 2 * sms) break;
    }
    return (int)best;
}

cudaError_t launch_cache_shared_rows(const CacheSharedArgs& a, cudaStream_t s)
{
    return a.shape.padded == 64 ? launch_rows<64>(a, s) : a.shape.padded == 128 ? launch_rows<128>(a, s) : launch_rows<256>(a, s);
}

cudaError_t launch_cache_shared_prefix(const CacheSharedArgs& a, cudaStream_t s)
{
    return a.shape.padded == 64 ? launch_prefix_of<64>(a, s) : a.shape.padded == 128 ? launch_prefix_of<128>(a, s) : launch_prefix_of<256>(a, s);
}

cudaError_t launch_cache_shared_join(const CacheSharedArgs& a, cudaStream_t s)
{
    return a.shape.padded == 64 ? launch_join<64>(a, s) : a.shape.padded == 128 ? launch_join<128>(a, s) : launch_join<256>(a, s);
}

}  // namespace lq
