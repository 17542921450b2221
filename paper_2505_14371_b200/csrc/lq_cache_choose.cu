// Bounds of a page's keys, and the pages that they choose for a sequence's queries.
//
// Bounds.  Coordinate d of the keys of a page lies in [lower_d, upper_d] * N / 127, whole numbers of 8 bits, N the largest norm: for a
// query q, sum_d max(q_d lower_d, q_d upper_d) is then at least every q . k of the page.  The extremes are those of the rows' values as
// they are read back (fp32 products of level and norm), times 127 fl(1 / N) and rounded outwards.
//
// Scores.  The query becomes whole numbers, too, and its positive and negative parts two operands: the sum above is then
// positive . upper + negative . lower, two byte products of four coordinates an instruction.  Sums of whole numbers do not hang on their order,
// so that a choice is the same on every path.  (Below 2^24: 256 * 127^2; as a float it is exact.)
//
// What bounds them.  Bounds: instructions (8 a pair of coordinates: look-up, products, extremes), 16384 tokens of 8 heads of 128 in 13 us with a cold
// cache, of which 1.5 would be the bytes'.  Choice: the chain of length, page numbers, bounds, queries and ranks, 10 to 18 us for 57 to 512 pages a
// sequence; the bounds of the first pages are asked for before the queries are turned.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

namespace cg = cooperative_groups;

namespace lq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr float kLeast = 7.8886090522101181e-31f;       // 2^-100: below, a norm or a query counts as 0
constexpr float kPart = 1.0f / 127.0f;

__device__ __forceinline__ bool counts(float largest) { return largest >= kLeast && largest < INFINITY; }

// ---- bounds --------------------------------------------------------------------------------------------------

// `split` warps take a page's rows of one head; a lane has 8 coordinates of every row of its own.  What a byte of a row stands for is looked up in shared
// memory, the two signed levels of symbols of 4 bits at once; a lane's copy of the table is in banks of its own (16 copies of two levels, 32 of one).
// Few pages are split over more warps, for their latency; many are not, as what a warp does behind its rows is half of what it does for 16 of them.
template <int P, int WK>
__global__ void __launch_bounds__(kThreads) bounds_kernel(const __grid_constant__ CacheBoundsArgs a, int split)
{
    constexpr int kLanes = P / 8, kRows = 32 / kLanes;
    extern __shared__ __align__(16) char smem[];
    float* const values = reinterpret_cast<float*>(smem);       // [256][32]
    float* const most = values + 256 * 32;                      // [kWarps][P], then least, then the norms
    float* const least = most + kWarps * P;
    float* const norms = least + kWarps * P;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    {
        auto level = [&](int symbol) { const float v = a.tables[LQ_KEYS].levels[symbol >> 1]; return symbol & 1 ? -v : v; };
        const int e = threadIdx.x;                              // a thread fills an entry, a warp's lanes at different banks
        const float x = level(WK == 4 ? e & 15 : e), y = WK == 4 ? level(e >> 4) : x;
        float4* row = reinterpret_cast<float4*>(values + 32 * e);
#pragma unroll
        for (int j = 0; j < 8; ++j) row[(j + lane) & 7] = make_float4(x, y, x, y);
    }
    static_assert(kThreads == 256, "a thread an entry");
    pdl_wait();
    pdl_launch_next();
    __syncthreads();
    const int per = kWarps / split, part = warp % split, page_size = 1 << a.shape.page_shift;
    const int row0 = lane / kLanes, col = lane % kLanes;
    const int64_t items = a.count * a.shape.heads;
    const char* const mine = reinterpret_cast<const char*>(values) + (WK == 4 ? (lane & 15) * 8 : lane * 4);
    for (int64_t first = (int64_t)blockIdx.x * per; first < items; first += (int64_t)gridDim.x * per) {
        const int64_t item = first + warp / split;
        int page = -1, head = 0;
        if (item < items) {
            const int64_t at = item / a.shape.heads;
            head = (int)(item - at * a.shape.heads);
            page = a.which[at];
            if (page >= a.num_pages) {
                if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_PAGE);
                page = -1;
            }
        }
        float up[8], down[8], n = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) { up[i] = -INFINITY; down[i] = INFINITY; }
        if (page >= 0) {
            const uint32_t* base = a.pages + (int64_t)page * a.shape.page_words + head * a.shape.head_words;
            const float* row_norms = reinterpret_cast<const float*>(base + ((a.shape.row_words[0] + a.shape.row_words[1]) << a.shape.page_shift));
            const uint32_t* codes = base + col * (WK / 4);
            const int end = (part + 1) * (page_size / split);
#pragma unroll 4
            for (int r = part * (page_size / split) + row0; r < end; r += kRows) {
                uint32_t w[WK / 4];
                if constexpr (WK == 8) {
                    const uint2 v = *reinterpret_cast<const uint2*>(codes + r * (P * WK / 32));
                    w[0] = v.x; w[WK / 4 - 1] = v.y;
                } else {
                    w[0] = codes[r * (P * WK / 32)];
                }
                const float norm = row_norms[r];
                n = norm >= 0.0f ? fmaxf(n, norm) : INFINITY;   // (NaN: no bounds)
                if constexpr (WK == 8) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v = __fmul_rn(norm, *reinterpret_cast<const float*>(mine + (__byte_perm(w[i / 4], 0, 0x4440 + i % 4) << 7)));
                        up[i] = fmaxf(up[i], v);
                        down[i] = fminf(down[i], v);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t at = (i == 0 ? w[0] << 7 : w[0] >> (8 * i - 7)) & (255u << 7);
                        const float2 l = *reinterpret_cast<const float2*>(mine + at);
                        const float x = __fmul_rn(norm, l.x), y = __fmul_rn(norm, l.y);
                        up[2 * i] = fmaxf(up[2 * i], x);
                        down[2 * i] = fminf(down[2 * i], x);
                        up[2 * i + 1] = fmaxf(up[2 * i + 1], y);
                        down[2 * i + 1] = fminf(down[2 * i + 1], y);
                    }
                }
            }
        }
#pragma unroll
        for (int o = kLanes; o < 32; o *= 2) {
            n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, o));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                up[i] = fmaxf(up[i], __shfl_xor_sync(0xffffffffu, up[i], o));
                down[i] = fminf(down[i], __shfl_xor_sync(0xffffffffu, down[i], o));
            }
        }
        if (split > 1) {
            if (lane < kLanes)
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    *reinterpret_cast<float4*>(most + warp * P + 8 * lane + i) = make_float4(up[i], up[i + 1], up[i + 2], up[i + 3]);
                    *reinterpret_cast<float4*>(least + warp * P + 8 * lane + i) = make_float4(down[i], down[i + 1], down[i + 2], down[i + 3]);
                }
            if (lane == 0) norms[warp] = n;
            __syncthreads();
            if (part == 0 && lane < kLanes)
                for (int w = warp + 1; w < warp + split; ++w) {
                    n = fmaxf(n, norms[w]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        up[i] = fmaxf(up[i], most[w * P + 8 * lane + i]);
                        down[i] = fminf(down[i], least[w * P + 8 * lane + i]);
                    }
                }
        }
        if (page >= 0 && part == 0 && lane < kLanes) {
            const float inv = counts(n) ? __fmul_rn(__frcp_rn(n), 127.0f) : 0.0f;
            auto packed = [&](const float (&v)[8], int i, bool above) {
                uint32_t w = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x = inv == 0.0f ? 0.0f : __fmul_rn(v[i + k], inv);
                    const int b = min(max(above ? __float2int_ru(x) : __float2int_rd(x), -127), 127);
                    w |= (uint32_t)(b & 255) << (8 * k);
                }
                return w;
            };
            uint32_t* const to = a.bounds + (int64_t)page * cache_bounds_words(a.shape.heads, P);
            *reinterpret_cast<uint2*>(to + head * (P / 2) + 2 * col) = make_uint2(packed(up, 0, true), packed(up, 4, true));
            *reinterpret_cast<uint2*>(to + head * (P / 2) + P / 4 + 2 * col) = make_uint2(packed(down, 0, false), packed(down, 4, false));
            if (col == 0) reinterpret_cast<float*>(to)[a.shape.heads * (P / 2) + head] = inv == 0.0f ? 0.0f : __fmul_rn(n, kPart);
        }
        if (split > 1) __syncthreads();
    }
}

template <int P, int WK>
cudaError_t launch_bounds(const CacheBoundsArgs& a, cudaStream_t s)
{
    constexpr int kBytes = 4 * (256 * 32 + kWarps * (2 * P + 1));
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = opt_in_shared_memory(configured, kBytes, bounds_kernel<P, WK>);
    // 16 rows a warp at least, and as few warps a page as keep the GPU's SMs busy
    const int64_t items = a.count * a.shape.heads;
    int split = 1;
    while (split < kWarps && split < 1 << (a.shape.page_shift - 4) && items * split < (int64_t)a.sms * 2 * kWarps) split *= 2;
    const int per = kWarps / split;
    const int64_t groups = (items + per - 1) / per, most = (int64_t)a.sms * 4;
    if (e == cudaSuccess) e = launch(bounds_kernel<P, WK>, (unsigned)(groups < most ? groups : most), kThreads, kBytes, s, a, split);
    return e;
}

// ---- choice --------------------------------------------------------------------------------------------------

constexpr int kBlock = 16;              // queries at a time
constexpr int kBins = 2048;
constexpr int kKeys = kCacheChooseKeys;
constexpr int kAhead = 4;               // pages that a group of lanes has under way

template <int P>
struct ChooseShared {
    alignas(16) uint8_t positive[kBlock][P], negative[kBlock][P];
    float per[kBlock];
    uint32_t low[kWarps], high[kWarps];
    uint2 sums[kWarps];
    uint32_t found[3];
    uint32_t bins[kBins];
    uint32_t keys[1];                   // kKeys or the table's pages, whichever is less
};

// A query's coordinate as it is stored, and as a number: what its bits mean is looked at when all loads are under way.
template <bool kFloat>
__device__ __forceinline__ uint32_t raw(const char* row, int d)
{
    if constexpr (kFloat) return reinterpret_cast<const uint32_t*>(row)[d];
    else return reinterpret_cast<const unsigned short*>(row)[d];
}
template <bool kFloat>
__device__ __forceinline__ float number(uint32_t v, int type)
{
    if constexpr (kFloat) return __uint_as_float(v);
    else return type == LQ_BF16 ? __uint_as_float(v << 16) : __half2float(__ushort_as_half((unsigned short)v));
}

// A score as a number whose order is the scores' (0 is kept for pages that are not there).
__device__ __forceinline__ uint32_t key_of(float score)
{
    const uint32_t b = __float_as_uint(score + 0.0f);           // (one zero)
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// Inclusive sums over the threads of a CTA.
__device__ __forceinline__ uint2 block_scan(uint2 v, uint2* sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) { v.x += x; v.y += y; }
    }
    __syncthreads();
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    for (int w = 0; w < warp; ++w) { v.x += sums[w].x; v.y += sums[w].y; }
    return v;
}

// A cluster of CTAs takes one (sequence, head): each scores its share of the pages, the first one chooses.
template <int P, bool kFloat>
__global__ void __launch_bounds__(kThreads) choose_kernel(const __grid_constant__ CacheChooseArgs a)
{
    constexpr int kLanes = P / 16, kGroups = kThreads / kLanes;
    extern __shared__ __align__(16) char smem[];
    ChooseShared<P>& sh = *reinterpret_cast<ChooseShared<P>*>(smem);
    const cg::cluster_group cluster = cg::this_cluster();
    const int ranks = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t item = blockIdx.x / ranks;
    const int sequence = (int)(item / a.shape.heads), head = (int)(item - (int64_t)sequence * a.shape.heads);
    pdl_wait();
    pdl_launch_next();
    const int64_t room = a.table_width << a.shape.page_shift;
    const int given = a.lengths[sequence];
    const int64_t length = given < 0 ? 0 : given > room ? room : given;
    if (given != length && rank == 0 && head == 0 && tid == 0) atomicOr(a.flags, LQ_CACHE_BAD_LENGTH);
    const int pages = (int)((length + (1 << a.shape.page_shift) - 1) >> a.shape.page_shift);
    const int32_t* const table = a.table + sequence * a.table_width;
    int32_t* const chosen = a.chosen + item * a.keep;
    if (rank == 0 && tid == 0) a.seen[item] = (int32_t)(length - ((int64_t)max(pages - a.keep, 0) << a.shape.page_shift));
    if (pages <= a.keep) {
        if (rank == 0)
            for (int i = tid; i < a.keep; i += kThreads) chosen[i] = i < pages ? table[i] : -1;
        return;
    }
    // scored are the pages first .. first + middle
    const int middle = pages - a.first - a.last, wanted = a.keep - a.first - a.last;
    const bool inside = middle <= kKeys;
    uint32_t* const keys = inside ? cluster.map_shared_rank(sh.keys, 0) : a.scores + item * a.table_width;
    if (inside && ranks > 1) cluster.sync();                    // (the first CTA has begun)
    const int share = (middle + ranks - 1) / ranks, begin = min(rank * share, middle), end = min(begin + share, middle);
    const int group = tid / kLanes, col = tid % kLanes;
    const int64_t page_words = cache_bounds_words(a.shape.heads, P);
    // bounds of kAhead pages of this thread's group of lanes: asked for before the queries are looked at
    uint4 up[kAhead], down[kAhead];
    float scale[kAhead];
    bool there[kAhead];
    auto fetch = [&](int base) {
        int page[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) { const int i = base + j * kGroups + group; page[j] = i < end ? table[a.first + i] : -1; }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            there[j] = page[j] >= 0 && page[j] < a.num_pages;
            up[j] = down[j] = make_uint4(0, 0, 0, 0);
            scale[j] = 0.0f;
            if (there[j]) {
                const uint32_t* from = a.bounds + page[j] * page_words;
                up[j] = *reinterpret_cast<const uint4*>(from + head * (P / 2) + 4 * col);
                down[j] = *reinterpret_cast<const uint4*>(from + head * (P / 2) + P / 4 + 4 * col);
                scale[j] = reinterpret_cast<const float*>(from)[a.shape.heads * (P / 2) + head];
            }
        }
    };
    for (int block = 0; block < a.group; block += kBlock) {
        const int queries = min(kBlock, a.group - block);
        fetch(begin);
        __syncthreads();
        for (int q = warp; q < queries; q += kWarps) {          // the queries as whole numbers
            const char* const row = static_cast<const char*>(a.queries.data) + (int64_t)sequence * a.queries.token_bytes +
                                    (int64_t)(head * a.group + block + q) * a.queries.head_bytes;
            const CacheRotary& r = a.rotary;
            const float* angles = r.table;
            bool lost = false;
            if (r.table) {
                const int64_t at = r.at ? r.at[sequence] : length - 1;
                lost = at < 0 || at >= r.positions;
                if (lost) { if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION); }
                else angles += at * r.dim;
            }
            uint32_t bits[P / 32], other[P / 32];
            float x[P / 32], c[P / 32], t[P / 32], top = 0.0f;
            const int half = r.dim / 2;
#pragma unroll
            for (int i = 0; i < P / 32; ++i) {
                const int d = lane + 32 * i;
                const bool turned = r.table && !lost && d < r.dim;
                bits[i] = d < a.shape.dim ? raw<kFloat>(row, d) : 0;
                other[i] = turned ? raw<kFloat>(row, r.interleaved ? d ^ 1 : d < half ? d + half : d - half) : 0;
                const int p = r.interleaved ? d / 2 : d < half ? d : d - half;
                c[i] = turned ? angles[p] : 1.0f;
                t[i] = turned ? angles[half + p] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < P / 32; ++i) {
                const int d = lane + 32 * i;
                x[i] = number<kFloat>(bits[i], a.queries.type);
                if (r.table && !lost && d < r.dim) {
                    const bool lower = r.interleaved ? d % 2 == 0 : d < half;
                    const float u = number<kFloat>(other[i], a.queries.type);
                    x[i] = lower ? __fsub_rn(__fmul_rn(x[i], c[i]), __fmul_rn(u, t[i])) : __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(u, t[i]));
                }
                top = fabsf(x[i]) <= top ? top : fabsf(x[i]);   // (keeps NaN)
                if (x[i] != x[i]) top = INFINITY;
            }
            top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
            const bool live = counts(top) && !lost;
            const float inv = live ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f;
#pragma unroll
            for (int i = 0; i < P / 32; ++i) {
                const int w = live ? __float2int_rn(__fmul_rn(x[i], inv)) : 0;
                sh.positive[q][lane + 32 * i] = (uint8_t)max(w, 0);
                sh.negative[q][lane + 32 * i] = (uint8_t)min(w, 0);
            }
            if (lane == 0) sh.per[q] = live ? __fmul_rn(top, kPart) : 0.0f;
        }
        __syncthreads();
        for (int base = begin; base < end; base += kGroups * kAhead) {
            float best[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) best[j] = -INFINITY;
            if (base > begin) fetch(base);
            for (int q = 0; q < queries; ++q) {
                const uint4 p = *reinterpret_cast<const uint4*>(&sh.positive[q][16 * col]);
                const uint4 n = *reinterpret_cast<const uint4*>(&sh.negative[q][16 * col]);
                const float per = sh.per[q];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    int dot = __dp4a((int)up[j].x, (int)p.x, 0);
                    dot = __dp4a((int)up[j].y, (int)p.y, dot);
                    dot = __dp4a((int)up[j].z, (int)p.z, dot);
                    dot = __dp4a((int)up[j].w, (int)p.w, dot);
                    dot = __dp4a((int)down[j].x, (int)n.x, dot);
                    dot = __dp4a((int)down[j].y, (int)n.y, dot);
                    dot = __dp4a((int)down[j].z, (int)n.z, dot);
                    dot = __dp4a((int)down[j].w, (int)n.w, dot);
#pragma unroll
                    for (int o = 1; o < kLanes; o *= 2) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    best[j] = fmaxf(best[j], __fmul_rn(__fmul_rn((float)dot, per), scale[j]));
                }
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = base + j * kGroups + group;
                if (col == 0 && i < end) {
                    const uint32_t key = there[j] ? key_of(best[j]) : 0;
                    keys[i] = block > 0 ? max(keys[i], key) : key;
                }
            }
        }
    }
    if (ranks > 1) cluster.sync(); else __syncthreads();
    if (rank > 0) return;

    const uint32_t* const mine = inside ? sh.keys : keys;
    auto ends = [&]() {                                         // the pages that are always kept
        for (int i = tid; i < a.first + a.last; i += kThreads)
            if (i < a.first) chosen[i] = table[i];
            else chosen[a.keep - a.last + (i - a.first)] = table[pages - a.last + (i - a.first)];
    };
    if (middle <= kThreads) {                                   // ---- a thread a page: how many stand before it (57 pages: 3 us less than by bins)
        const uint32_t k = tid < middle ? mine[tid] : 0;
        int before = 0;
#pragma unroll 4
        for (int i = 0; i < middle; ++i) { const uint32_t other = mine[i]; before += other > k || (other == k && i < tid); }
        const bool taken = tid < middle && before < wanted;
        const uint32_t votes = __ballot_sync(0xffffffffu, taken);
        if (lane == 0) sh.low[warp] = __popc(votes);
        __syncthreads();
        int at = __popc(votes & ((1u << lane) - 1));
        for (int w = 0; w < warp; ++w) at += sh.low[w];
        if (taken) chosen[a.first + at] = table[a.first + tid];
        ends();
        return;
    }
    // ---- the `wanted` largest keys: bins over the range that is left, until the last one is taken whole or is one number
    uint32_t low = 0xffffffffu, high = 0;
    for (int i = tid; i < middle; i += kThreads) { const uint32_t k = mine[i]; low = min(low, k); high = max(high, k); }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    if (lane == 0) { sh.low[warp] = low; sh.high[warp] = high; }
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) { low = min(low, sh.low[w]); high = max(high, sh.high[w]); }
    uint32_t left = (uint32_t)wanted;                           // to be taken from [low, high]; what is above is taken
    bool all = left == (uint32_t)middle;
    while (!all && left > 0 && low != high) {
        const int shift = max(0, 32 - __clz(high - low) - 11);
        for (int i = tid; i < kBins; i += kThreads) sh.bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < middle; i += kThreads) {
            const uint32_t k = mine[i];
            if (k >= low && k <= high) atomicAdd(&sh.bins[(k - low) >> shift], 1u);
        }
        __syncthreads();
        // from the top: thread t has bins kBins - 1 - 8 t and down
        constexpr int kOwn = kBins / kThreads;
        uint32_t own = 0;
        for (int i = 0; i < kOwn; ++i) own += sh.bins[kBins - 1 - kOwn * tid - i];
        const uint32_t to = block_scan(make_uint2(own, 0), sh.sums).x;
        if (to >= left && to - own < left) {
            uint32_t above = to - own;
            int b = kBins - 1 - kOwn * tid;
            while (above + sh.bins[b] < left) above += sh.bins[b--];
            sh.found[0] = (uint32_t)b; sh.found[1] = left - above; sh.found[2] = sh.bins[b] == left - above;
        }
        __syncthreads();
        low += sh.found[0] << shift;
        high = min(high, low + ((1u << shift) - 1));
        left = sh.found[1];
        all = sh.found[2] != 0;
        __syncthreads();
    }

    // ---- in their order: a thread goes through a run of pages
    const int run = (middle + kThreads - 1) / kThreads, from = min(tid * run, middle), until = min(from + run, middle);
    uint2 count = make_uint2(0, 0);
    for (int i = from; i < until; ++i) {
        const uint32_t k = mine[i];
        count.x += k > high;
        count.y += k >= low && k <= high;
    }
    const uint2 upto = block_scan(count, sh.sums);
    uint32_t sure = upto.x - count.x, even = upto.y - count.y;  // of the pages before
    for (int i = from; i < until; ++i) {
        const uint32_t k = mine[i];
        const bool above = k > high, level = k >= low && k <= high;
        if (above || (level && (all || even < left))) chosen[a.first + sure + (all ? even : min(even, left))] = table[a.first + i];
        sure += above;
        even += level;
    }
    ends();
}

template <int P, bool kFloat>
cudaError_t launch_choose_as(const CacheChooseArgs& a, cudaStream_t s)
{
    const int64_t items = (int64_t)a.batch * a.shape.heads;
    // more CTAs an item while the GPU has room for them and each has pages to score
    unsigned ranks = 1;
    while (ranks < 8 && items * ranks * 2 <= a.sms && (int64_t)ranks * 128 <= a.table_width) ranks *= 2;
    const int keys = (int)(a.table_width < kKeys ? a.table_width : kKeys), bytes = (int)sizeof(ChooseShared<P>) + 4 * keys;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e = opt_in_shared_memory(configured, (int)sizeof(ChooseShared<P>) + 4 * kKeys, choose_kernel<P, kFloat>);
    if (e == cudaSuccess) e = launch_cluster(choose_kernel<P, kFloat>, (unsigned)(items * ranks), kThreads, bytes, ranks, s, a);
    return e;
}

template <int P>
cudaError_t launch_choose(const CacheChooseArgs& a, cudaStream_t s)
{
    return a.queries.type == LQ_F32 ? launch_choose_as<P, true>(a, s) : launch_choose_as<P, false>(a, s);
}

}  // namespace

cudaError_t launch_cache_bounds(const CacheBoundsArgs& a, cudaStream_t s)
{
    const bool fine = a.shape.sym_bits[0] == 8;
    if (a.shape.padded == 64) return fine ? launch_bounds<64, 8>(a, s) : launch_bounds<64, 4>(a, s);
    if (a.shape.padded == 128) return fine ? launch_bounds<128, 8>(a, s) : launch_bounds<128, 4>(a, s);
    return fine ? launch_bounds<256, 8>(a, s) : launch_bounds<256, 4>(a, s);
}

cudaError_t launch_cache_choose(const CacheChooseArgs& a, cudaStream_t s)
{
    return a.shape.padded == 64 ? launch_choose<64>(a, s) : a.shape.padded == 128 ? launch_choose<128>(a, s) : launch_choose<256>(a, s);
}

}  // namespace lq
