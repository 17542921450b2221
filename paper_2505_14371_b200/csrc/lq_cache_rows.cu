// Rows of the key-value cache: quantised as they are written, and read back.
//
// A lane takes 8 coordinates of a row (token, head, keys or values) at a time: 16 bytes of fp16 or bf16 in one load or store, one
// 32-bit word of 4-bit symbols (or two of 8-bit ones), two Philox blocks.  The writing kernel gives a lane two such parts of rows of 128
// and 256 (lane i those from 8 i and from padded / 2 + 8 i): with one, what a row costs besides its coordinates was a third of the
// instructions (16384 tokens of 8 heads of 128 65 us, 42 with two); rows of 64 have one (9600 tokens of 10 heads of 41, unbiased: 36 us, 38 with two).
// A row's norm is an all-reduce over its lanes, its symbols are found by one look-up each (CacheSearch).
//
// What bounds them.  Writing: instructions, some 32 a coordinate (rotation 15 of a key's, look-up and packing 14, norm 4), at 70 %
// of the issue slots; 76 MB read and 18 MB written in 42 us.  Reading: its writes, 3.7 TB/s beside 1 TB/s of reads (100 003 tokens in
// 112 us; a plain fill writes 3.9 TB/s).  Few tokens: latency of slot -> row -> norm -> store, and the host.
//
// Both kernels start beside their predecessor, which may be what writes their slots, rows, positions or pages (a row is read back right
// after it was written): all that is read behind pdl_wait is read by ordinary loads, never through the read-only path.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstddef>
#include <type_traits>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

namespace lq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kEach = 8;                // coordinates at a time
template <int P>
constexpr int kPartsOf = P >= 128 ? 2 : 1;      // ... of a lane of the writing kernel
constexpr int kWriteCtas = 3;           // CTAs of the writing kernel that an SM holds at once, by its registers

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T of_f32(float v);
template <> __device__ __forceinline__ float of_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half of_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 of_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Coordinates d .. d+7 of a row, zeros past its end.  `wide`: the row starts on a 16-byte boundary.
template <typename T>
struct alignas(16) Eight { T v[kEach]; };

template <typename T>
__device__ __forceinline__ Eight<T> load8(const T* row, int d, int dim, bool wide)
{
    Eight<T> e;
    if (wide && d + kEach <= dim) {
#pragma unroll
        for (int i = 0; i < (int)(kEach * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(&e)[i] = __ldca(reinterpret_cast<const uint4*>(row + d) + i);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) e.v[i] = d + i < dim ? row[d + i] : of_f32<T>(0.0f);
    }
    return e;
}

template <typename T>
__device__ __forceinline__ void floats(float (&x)[kEach], const Eight<T>& e)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {   // the upper half of a float: one instruction each
#pragma unroll
        for (int i = 0; i < kEach; i += 2) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(&e)[i / 2];
            x[i] = __uint_as_float(w << 16);
            x[i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = to_f32(e.v[i]);
    }
}

template <typename T>
__device__ __forceinline__ void store8(const float (&x)[kEach], T* row, int d, int dim, bool wide)
{
    if (wide && d + kEach <= dim) {
        constexpr int kWords = kEach * sizeof(T) / 16;
        alignas(16) T t[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) t[i] = of_f32<T>(x[i]);
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(row + d)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) if (d + i < dim) row[d + i] = of_f32<T>(x[i]);
    }
}

__device__ __forceinline__ void load_angles(float* to, const float* from, int n)
{
    for (int i = 0; i < n; i += 4) *reinterpret_cast<float4*>(to + i) = __ldca(reinterpret_cast<const float4*>(from + i));
}

// The pairs of the first `dim` coordinates turned by the angles of `position`.  x holds coordinates d .. d+7 of `row`; the
// partners that this lane does not hold come from the row again (the first level cache has it).
template <typename T>
__device__ __forceinline__ void rotate8(float (&x)[kEach], const T* row, int d, const CacheRotary& r, const float* angles, int64_t position, bool wide)
{
    const float* c = angles + (int64_t)(uint32_t)position * r.dim;
    const float* s = c + r.dim / 2;
    if (r.wide && wide) {
        if (d >= r.dim) return;
        alignas(16) float cc[kEach], ss[kEach];
        if (r.interleaved) {
            load_angles(cc, c + d / 2, kEach / 2);
            load_angles(ss, s + d / 2, kEach / 2);
#pragma unroll
            for (int i = 0; i < kEach; i += 2) {
                const float a = x[i], b = x[i + 1];
                x[i] = __fsub_rn(__fmul_rn(a, cc[i / 2]), __fmul_rn(b, ss[i / 2]));
                x[i + 1] = __fadd_rn(__fmul_rn(b, cc[i / 2]), __fmul_rn(a, ss[i / 2]));
            }
            return;
        }
        const int half = r.dim / 2;
        const bool first = d < half;
        const int p = first ? d : d - half;
        float y[kEach];
        floats(y, load8(row, first ? d + half : p, r.dim, true));
        load_angles(cc, c + p, kEach);
        load_angles(ss, s + p, kEach);
        const uint32_t flip = first ? 0x80000000u : 0u;                 // (a product's sign is exact)
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = __fadd_rn(__fmul_rn(x[i], cc[i]), __fmul_rn(__uint_as_float(__float_as_uint(y[i]) ^ flip), ss[i]));
        return;
    }
    if (r.interleaved) {
#pragma unroll
        for (int i = 0; i < kEach; i += 2) {
            if (d + i < r.dim) {
                const float cc = __ldca(c + (d + i) / 2), ss = __ldca(s + (d + i) / 2), a = x[i], b = x[i + 1];
                x[i] = __fsub_rn(__fmul_rn(a, cc), __fmul_rn(b, ss));
                x[i + 1] = __fadd_rn(__fmul_rn(b, cc), __fmul_rn(a, ss));
            }
        }
    } else {
        const int half = r.dim / 2;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = d + i;
            if (e < r.dim) {
                const bool first = e < half;
                const int p = first ? e : e - half;
                const float cc = __ldca(c + p), ss = __ldca(s + p), other = to_f32(row[first ? e + half : p]);
                x[i] = first ? __fsub_rn(__fmul_rn(x[i], cc), __fmul_rn(other, ss))
                             : __fadd_rn(__fmul_rn(x[i], cc), __fmul_rn(other, ss));
            }
        }
    }
}

// N as the cache keeps it (0: the row is kept as zeros); bad: NaN, Inf or a norm that overflows.  Same value in all lanes.
template <int kLanes, int kParts>
__device__ __forceinline__ float row_norm(const float (&x)[kParts][kEach], int q, bool& bad)
{
    float n;
    if (q == 0) {
        // the maximum drops NaN: a sum of x * 0 keeps it, and Inf
        float m = 0.0f, z = 0.0f;
#pragma unroll
        for (int c = 0; c < kParts; ++c)
#pragma unroll
            for (int i = 0; i < kEach; ++i) { m = fmaxf(m, fabsf(x[c][i])); z = fmaf(x[c][i], 0.0f, z); }
        if (z != 0.0f) m = INFINITY;
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        n = m;
    } else {
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < kParts; ++c)
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const double a = fabs((double)x[c][i]);
                sum = q == 1 ? sum + a : fma(a, a, sum);
            }
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        n = (float)(q == 1 ? sum : sqrt(sum));
    }
    bad = !(n <= 3.402823466e38f);
    return bad || n < 1.17549435e-38f ? 0.0f : n;
}

// The (token, head) pair of this group of lanes and where its slot is.
struct Place {
    int64_t slot;
    int token, head;
};

__device__ __forceinline__ Place place_of(uint32_t r, int heads, const CacheRowsOf& by, const int64_t* slots)
{
    Place p;
    const uint32_t token = __umulhi(2 * r, by.factor) >> by.shift;
    p.token = (int)token;
    p.head = (int)(r - token * heads);
    p.slot = __ldca(slots + token);
    return p;
}

// What a kernel of rows keeps of the level tables.
struct SharedSearch {
    CacheSearch search;
    float2 low_gap[kCacheLevels];       // a level and the gap above it
};

// Symbols 2 * index + sign of 8 coordinates, packed as the row has them (hi: the upper four of 8 bits).
template <bool kUnbiased>
__device__ __forceinline__ void symbols8(const float (&x)[kEach], float norm, float inv, int bits, const SharedSearch& t, const uint32_t (&rnd)[kEach],
                                         uint32_t& lo, uint32_t& hi)
{
    uint32_t at[kEach];
    if (t.search.entries) {
        // (a number just above 1 is in the bin of 1; NaN, in a row that is kept as zeros, becomes `lowest`)
        const uint32_t* entry = t.search.entry - t.search.first;
        const int shift = t.search.shift;
        const float lowest = t.search.lowest;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t pattern = __float_as_uint(fmaxf(__fmul_rn(fabsf(x[i]), inv), lowest));
            at[i] = (entry[pattern >> shift] + pattern) >> shift;
        }
    } else {
        const int steps = t.search.steps;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float u = fminf(__fmul_rn(fabsf(x[i]), inv), 1.0f);
            // 4096 + u has round(2048 u) in its last bits
            at[i] = t.search.start[__float_as_uint(__fadd_rn(u, 4096.0f)) - 0x45800000u];
            for (int s = 0; s < steps; ++s) at[i] += u >= t.search.edge[at[i] + 1] ? 1 : 0;
        }
    }
    if (kUnbiased) {                    // whether the upper neighbour is taken
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float u = fminf(__fmul_rn(fabsf(x[i]), inv), 1.0f);
            const float2 lg = t.low_gap[at[i]];
            at[i] += __fmul_rn(__fmul_rn((float)(rnd[i] >> 9), 1.1920928955078125e-7f), lg.y) < __fsub_rn(u, lg.x) ? 1 : 0;
        }
    }
    lo = hi = 0;
    if (bits == 4) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            lo += at[i] << (4 * i + 1);
            if (x[i] < 0.0f) lo += 1u << (4 * i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo += at[i] << (8 * i + 1);
            hi += at[4 + i] << (8 * i + 1);
            if (x[i] < 0.0f) lo += 1u << (8 * i);
            if (x[4 + i] < 0.0f) hi += 1u << (8 * i);
        }
    }
    if (!(norm > 0.0f)) lo = hi = 0;
}

// Every CTA has its share of the keys, which are rotated, and then of the values.  Rows are fetched a round ahead.
template <typename T, int P, bool kUnbiased>
__global__ void __launch_bounds__(kRowThreads, kWriteCtas) cache_write_kernel(const __grid_constant__ CacheWriteArgs a)
{
    constexpr int kParts = kPartsOf<P>, kLanes = P / (kEach * kParts);
    __shared__ SharedSearch tables[2];
#pragma unroll 1
    for (int kind = 0; kind < 2; ++kind) {
        const CacheTable& t = a.tables[kind];
        const CacheSearch& s = kUnbiased ? t.floor : t.nearest;
        // the head, and the table of one of the two searches
        uint4* to = reinterpret_cast<uint4*>(&tables[kind].search);
        const uint4* from = reinterpret_cast<const uint4*>(&s);
        constexpr int kHead = (int)offsetof(CacheSearch, edge) / 16, kEntry = (int)offsetof(CacheSearch, entry) / 16;
        static_assert(offsetof(CacheSearch, edge) % 16 == 0 && offsetof(CacheSearch, entry) % 16 == 0, "parts are copied by 16 bytes");
        const int entries = s.entries, begin = entries ? kEntry : kHead, end = entries ? kEntry + (entries + 3) / 4 : kEntry;
        if (threadIdx.x < kHead) to[threadIdx.x] = from[threadIdx.x];
        for (int i = begin + threadIdx.x; i < end; i += kRowThreads) to[i] = from[i];
        if (kUnbiased)
            for (int i = threadIdx.x; i < kCacheLevels - 1; i += kRowThreads) {
                const float l = t.levels[i];
                tables[kind].low_gap[i] = make_float2(l, __fsub_rn(t.levels[i + 1], l));
            }
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_next();

    constexpr int kRows = kRowThreads / kLanes;
    const uint32_t rows = (uint32_t)(a.tokens * a.shape.heads), stride = gridDim.x * kRows, group = threadIdx.x / kLanes;
    const int lane = threadIdx.x % kLanes, page_size = 1 << a.shape.page_shift;
    auto from = [&](int part) { return (part * kLanes + lane) * kEach; };        // first coordinate of a part
    const bool turned = a.rotary.table != nullptr;
    const int64_t* const slots = fresh(a.slots);
    const int64_t* const positions = fresh(a.rotary.at);
    const float* const angles = fresh(a.rotary.table);
#pragma unroll 1
    for (int kind = 0; kind < 2; ++kind) {
        const SharedSearch& table = tables[kind];
        const int bits = a.shape.sym_bits[kind];
        const int codes_at = kind ? page_size * a.shape.row_words[0] : 0, row_words = a.shape.row_words[kind];
        const int norms_at = page_size * (a.shape.row_words[0] + a.shape.row_words[1] + kind);
        const char* const data = fresh(static_cast<const char*>(a.rows[kind].data));
        const int token_bytes = a.rows[kind].token_bytes, head_bytes = a.rows[kind].head_bytes;
        const bool wide = a.rows[kind].wide;

        int64_t next_slot = -1, next_position = 0;
        int next_head = 0;
        const T* next_row = nullptr;
        Eight<T> next[kParts] = {};
        auto fetch = [&](uint32_t r) {
            next_slot = -1;
            if (r >= rows) return;
            const Place p = place_of(r, a.shape.heads, a.by_head, slots);
            next_slot = p.slot; next_head = p.head;
            next_row = reinterpret_cast<const T*>(data + (int64_t)p.token * token_bytes + (int64_t)p.head * head_bytes);
#pragma unroll
            for (int c = 0; c < kParts; ++c) next[c] = load8(next_row, from(c), a.shape.dim, wide);
            if (turned) next_position = __ldca(positions + p.token);
        };
        fetch(blockIdx.x * kRows + group);
        for (uint32_t first = blockIdx.x * kRows; first < rows; first += stride) {
            // every lane of a warp takes part in the reductions, those without a row with whatever they hold
            int64_t slot = next_slot;
            const int64_t position = next_position;
            const int head = next_head;
            const T* const row = next_row;
            float x[kParts][kEach];
#pragma unroll
            for (int c = 0; c < kParts; ++c) floats(x[c], next[c]);
            fetch(first + stride + group);
            if (slot >= a.num_slots) { slot = -1; if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_SLOT); }
            if (turned && slot >= 0) {
                if ((uint64_t)position >= (uint64_t)a.rotary.positions) {
                    slot = -1;
                    if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION);
                } else if (kind == LQ_KEYS) {
#pragma unroll
                    for (int c = 0; c < kParts; ++c) {
                        rotate8(x[c], row, from(c), a.rotary, angles, position, wide);
                        asm volatile("" ::: "memory");                  // (the angles of one part at a time: registers)
                    }
                }
            }
            bool bad;
            const float norm = row_norm<kLanes, kParts>(x, a.shape.q, bad);
            if (slot < 0) continue;
            const float inv = norm > 0.0f ? __frcp_rn(norm) : 0.0f;
            const int place = (int)slot & (page_size - 1);
            uint32_t* base = a.pages + (int64_t)((uint32_t)slot >> a.shape.page_shift) * a.shape.page_words + head * a.shape.head_words;
            uint32_t* codes = base + codes_at + place * row_words;
#pragma unroll
            for (int c = 0; c < kParts; ++c) {
                uint32_t rnd[kEach];
                if (kUnbiased) {
                    const uint32_t c0 = (uint32_t)(head * a.shape.padded + from(c)) / 4;
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        philox4x32_10(c0 + j, 2 * a.layer + kind, (uint32_t)slot, a.step, a.seed_lo, a.seed_hi, w);
#pragma unroll
                        for (int i = 0; i < 4; ++i) rnd[4 * j + i] = w[i];
                    }
                }
                uint32_t lo, hi;
                symbols8<kUnbiased>(x[c], norm, inv, bits, table, rnd, lo, hi);
                if (bits == 4) codes[c * kLanes + lane] = lo;
                else reinterpret_cast<uint2*>(codes)[c * kLanes + lane] = make_uint2(lo, hi);
            }
            if (lane == 0) {
                reinterpret_cast<float*>(base)[norms_at + place] = norm;
                if (bad) atomicOr(a.flags, LQ_CACHE_NONFINITE);
            }
        }
    }
}

template <typename T, int kLanes>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ CacheReadArgs a)
{
    // signed levels by symbol: 16 of them lie in 16 banks, so that no look-up of 4-bit symbols has a conflict
    __shared__ float values[2][kCachePairs];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
        if (threadIdx.x < 1u << a.shape.sym_bits[kind]) {
            const float l = a.tables[kind].levels[threadIdx.x / 2];
            values[kind][threadIdx.x] = threadIdx.x % 2 ? -l : l;
        }
    __syncthreads();
    pdl_wait();
    pdl_launch_next();

    constexpr int kRows = kRowThreads / kLanes;
    const uint32_t rows = (uint32_t)(a.tokens * a.shape.heads);
    const int lane = threadIdx.x % kLanes, d = lane * kEach, page_size = 1 << a.shape.page_shift;
    const int64_t* const slots = fresh(a.slots);
    const uint32_t* const pages = fresh(a.pages);
    for (uint32_t r = blockIdx.x * kRows + threadIdx.x / kLanes; r < rows; r += gridDim.x * kRows) {
        Place p = place_of(r, a.shape.heads, a.by_head, slots);
        if (p.slot >= a.num_slots) { p.slot = -1; if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_SLOT); }
        const int place = (int)p.slot & (page_size - 1);
        const uint32_t* base = pages + (int64_t)((uint32_t)p.slot >> a.shape.page_shift) * a.shape.page_words + p.head * a.shape.head_words;
        uint2 w[2] = {};
        float norm[2] = {0.0f, 0.0f};
        if (p.slot >= 0) {
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const uint32_t* codes = base + (kind ? page_size * a.shape.row_words[0] : 0) + place * a.shape.row_words[kind];
                norm[kind] = __ldca(reinterpret_cast<const float*>(base + page_size * (a.shape.row_words[0] + a.shape.row_words[1])) +
                                    kind * page_size + place);
                if (a.shape.sym_bits[kind] == 4) w[kind].x = __ldca(codes + lane);
                else w[kind] = __ldca(reinterpret_cast<const uint2*>(codes) + lane);
            }
        }
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            float x[kEach];
            if (p.slot < 0) {
#pragma unroll
                for (int i = 0; i < kEach; ++i) x[i] = 0.0f;
            } else if (a.shape.sym_bits[kind] == 4) {
#pragma unroll
                for (int i = 0; i < kEach; ++i) x[i] = __fmul_rn(values[kind][w[kind].x >> (4 * i) & 15], norm[kind]);
            } else {
#pragma unroll
                for (int i = 0; i < kEach; ++i) x[i] = __fmul_rn(values[kind][(i < 4 ? w[kind].x : w[kind].y) >> (8 * (i & 3)) & 255], norm[kind]);
            }
            const CacheRows& out = a.rows[kind];
            store8(x, reinterpret_cast<T*>(static_cast<char*>(out.data) + (int64_t)p.token * out.token_bytes + (int64_t)p.head * out.head_bytes), d, a.shape.dim, out.wide);
        }
    }
}

__global__ void cache_clear_kernel(uint32_t* flags, uint32_t seen) { atomicAnd(flags, ~seen); }

// CTAs: as many as the rows need with `each` coordinates a lane, at most as the GPU holds at once (`resident` an SM).
template <typename Args, typename Go>
cudaError_t by_type_and_size(const Args& a, int each, int resident, Go go)
{
    const int lanes = a.shape.padded / each, type = a.rows[0].type;
    const int64_t blocks = (a.tokens * a.shape.heads * lanes + kRowThreads - 1) / kRowThreads;
    const unsigned grid = (unsigned)(blocks < resident * kSms ? blocks : resident * kSms);
    auto sized = [&](auto t) {
        if (a.shape.padded == 64) return go(t, std::integral_constant<int, 64>(), grid);
        if (a.shape.padded == 128) return go(t, std::integral_constant<int, 128>(), grid);
        return go(t, std::integral_constant<int, 256>(), grid);
    };
    return type == LQ_F32 ? sized(float()) : type == LQ_F16 ? sized(__half()) : sized(__nv_bfloat16());
}

}  // namespace

cudaError_t launch_cache_write(const CacheWriteArgs& a, cudaStream_t s)
{
    return by_type_and_size(a, a.shape.padded >= 128 ? kEach * kPartsOf<128> : kEach * kPartsOf<64>, kWriteCtas, [&](auto t, auto padded, unsigned grid) {
        using T = decltype(t);
        constexpr int P = decltype(padded)::value;
        return a.unbiased ? launch(cache_write_kernel<T, P, true>, grid, kRowThreads, 0, s, a)
                          : launch(cache_write_kernel<T, P, false>, grid, kRowThreads, 0, s, a);
    });
}

cudaError_t launch_cache_clear(uint32_t* flags, uint32_t seen)
{
    return launch_as(false, cache_clear_kernel, 1, 1, 0, 1, nullptr, flags, seen);
}

cudaError_t launch_cache_read(const CacheReadArgs& a, cudaStream_t s)
{
    return by_type_and_size(a, kEach, 8, [&](auto t, auto padded, unsigned grid) {
        return launch(cache_read_kernel<decltype(t), decltype(padded)::value / kEach>, grid, kRowThreads, 0, s, a);
    });
}

}  // namespace lq
