// Rows of the key-value cache: quantised as they are written, and read back.
//
// A row (token, head, keys or values) of `padded` coordinates is taken by padded / 8 lanes, 8 coordinates each: 16 bytes of
// fp16 or bf16 input in one load, one 32-bit word of 4-bit symbols (or two of 8-bit ones) in one store, two Philox blocks.
// Its norm is an all-reduce over those lanes.  Bound: the bytes of the rows on one side and of the page on the other; for
// few tokens the latency of slot -> row -> norm -> store.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

namespace lq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kEach = 8;                // coordinates a lane

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
__device__ __forceinline__ void load8(float (&x)[kEach], const T* row, int d, int dim, bool wide)
{
    if (wide && d + kEach <= dim) {
        constexpr int kWords = kEach * sizeof(T) / 16;
        alignas(16) T t[kEach];
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(t)[i] = __ldg(reinterpret_cast<const uint4*>(row + d) + i);
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = to_f32(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = d + i < dim ? to_f32(row[d + i]) : 0.0f;
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

// The pairs of the first `dim` coordinates turned by the angles of `position`.  x holds coordinates d .. d+7 of `row`; the
// partners that this lane does not hold come from the row again (the first level cache has it).
template <typename T>
__device__ __forceinline__ void rotate8(float (&x)[kEach], const T* row, int d, const CacheRotary& r, int64_t position)
{
    const float* c = r.table + position * r.dim;
    const float* s = c + r.dim / 2;
    if (r.interleaved) {
#pragma unroll
        for (int i = 0; i < kEach; i += 2) {
            if (d + i < r.dim) {
                const float cc = __ldg(c + (d + i) / 2), ss = __ldg(s + (d + i) / 2), a = x[i], b = x[i + 1];
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
                const float cc = __ldg(c + p), ss = __ldg(s + p), other = to_f32(row[first ? e + half : p]);
                x[i] = first ? __fsub_rn(__fmul_rn(x[i], cc), __fmul_rn(other, ss))
                             : __fadd_rn(__fmul_rn(x[i], cc), __fmul_rn(other, ss));
            }
        }
    }
}

// N as the cache keeps it (0: the row is kept as zeros); bad: NaN, Inf or a norm that overflows.  Same value in all lanes.
template <int kLanes>
__device__ __forceinline__ float row_norm(const float (&x)[kEach], int q, bool& bad)
{
    float n;
    if (q == 0) {
        uint32_t m = 0;                 // magnitudes order as their bit patterns; Inf and NaN come last
#pragma unroll
        for (int i = 0; i < kEach; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        n = __uint_as_float(m);
    } else {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const double a = fabs((double)x[i]);
            sum = q == 1 ? sum + a : fma(a, a, sum);
        }
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        n = (float)(q == 1 ? sum : sqrt(sum));
    }
    bad = !(n <= 3.402823466e38f);
    return bad || n < 1.17549435e-38f ? 0.0f : n;
}

template <typename T, int kLanes>
__global__ void __launch_bounds__(kRowThreads) cache_write_kernel(const __grid_constant__ CacheWriteArgs a)
{
    const int64_t thread = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int64_t rows = a.tokens * 2 * a.shape.heads;
    const int64_t r = thread / kLanes;
    const int lane = (int)(thread % kLanes), d = lane * kEach;
    // every lane of a warp takes part in the reductions, those past the last row with zeros
    const int64_t token = r < rows ? r / (2 * a.shape.heads) : 0;
    const int within = r < rows ? (int)(r - token * 2 * a.shape.heads) : 0;
    const int kind = within >= a.shape.heads, head = within - kind * a.shape.heads;
    int64_t slot = -1, position = 0;
    if (r < rows) {
        slot = __ldg(a.slots + token);
        if (a.rotary.table) position = __ldg(a.rotary.at + token);
        if (slot >= a.num_slots) { slot = -1; if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_SLOT); }
        if (slot >= 0 && a.rotary.table && (position < 0 || position >= a.rotary.positions)) {
            slot = -1;
            if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_POSITION);
        }
    }
    const bool live = slot >= 0;

    float x[kEach] = {};
    if (live) {
        const CacheRows& in = a.rows[kind];
        const T* row = static_cast<const T*>(in.data) + token * in.token_stride + head * in.head_stride;
        load8(x, row, d, a.shape.dim, in.wide);
        if (kind == LQ_KEYS && a.rotary.table) rotate8(x, row, d, a.rotary, position);
    }
    bool bad;
    const float norm = row_norm<kLanes>(x, a.shape.q, bad);
    if (!live) return;
    if (bad && lane == 0) atomicOr(a.flags, LQ_CACHE_NONFINITE);

    const float inv = norm > 0.0f ? __fdiv_rn(1.0f, norm) : 0.0f;
    const int bits = a.shape.sym_bits[kind], last = (1 << (bits - 1)) - 2;      // index of the last interval
    const float* levels = a.tables[kind].levels;
    uint32_t rnd[kEach];
    if (a.unbiased) {
        const uint32_t c0 = (uint32_t)(head * a.shape.padded + d) / 4;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            philox4x32_10(c0 + j, 2 * a.layer + kind, (uint32_t)slot, a.step, a.seed_lo, a.seed_hi, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) rnd[4 * j + i] = w[i];
        }
    }
    uint32_t sym[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const float u = norm > 0.0f ? fminf(__fmul_rn(fabsf(x[i]), inv), 1.0f) : 0.0f;
        int at = 0;
        for (int step = (last + 2) / 2; step > 0; step /= 2) {
            const int t = at + step;
            if (t <= last && __ldg(levels + t) <= u) at = t;
        }
        const float low = __ldg(levels + at), gap = __fsub_rn(__ldg(levels + at + 1), low);
        const float rho = a.unbiased ? __fmul_rn((float)(rnd[i] >> 9), 1.1920928955078125e-7f) : 0.5f;
        at += __fmul_rn(rho, gap) < __fsub_rn(u, low);
        sym[i] = norm > 0.0f ? 2 * at + (x[i] < 0.0f) : 0;
    }

    const int64_t page = slot >> a.shape.page_shift, place = slot & ((1 << a.shape.page_shift) - 1);
    const int64_t page_size = (int64_t)1 << a.shape.page_shift;
    uint32_t* base = a.pages + page * a.shape.page_words + head * a.shape.head_words;
    uint32_t* codes = base + (kind ? page_size * a.shape.row_words[0] : 0) + place * a.shape.row_words[kind];
    if (bits == 4) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) w |= sym[i] << (4 * i);
        codes[lane] = w;
    } else {
        uint2 w = make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w.x |= sym[i] << (8 * i); w.y |= sym[4 + i] << (8 * i); }
        reinterpret_cast<uint2*>(codes)[lane] = w;
    }
    if (lane == 0) {
        float* norms = reinterpret_cast<float*>(base + page_size * (a.shape.row_words[0] + a.shape.row_words[1]));
        norms[kind * page_size + place] = norm;
    }
}

template <typename T, int kLanes>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ CacheReadArgs a)
{
    const int64_t thread = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int64_t r = thread / kLanes;
    if (r >= a.tokens * 2 * a.shape.heads) return;
    const int lane = (int)(thread % kLanes), d = lane * kEach;
    const int64_t token = r / (2 * a.shape.heads);
    const int within = (int)(r - token * 2 * a.shape.heads);
    const int kind = within >= a.shape.heads, head = within - kind * a.shape.heads;
    int64_t slot = __ldg(a.slots + token);
    if (slot >= a.num_slots) { slot = -1; if (lane == 0) atomicOr(a.flags, LQ_CACHE_BAD_SLOT); }

    float x[kEach] = {};
    if (slot >= 0) {
        const int64_t page = slot >> a.shape.page_shift, place = slot & ((1 << a.shape.page_shift) - 1);
        const int64_t page_size = (int64_t)1 << a.shape.page_shift;
        const uint32_t* base = a.pages + page * a.shape.page_words + head * a.shape.head_words;
        const uint32_t* codes = base + (kind ? page_size * a.shape.row_words[0] : 0) + place * a.shape.row_words[kind];
        const float norm = __ldg(reinterpret_cast<const float*>(base + page_size * (a.shape.row_words[0] + a.shape.row_words[1])) +
                                 kind * page_size + place);
        const uint32_t* pairs = a.tables[kind].pairs;
        if (a.shape.sym_bits[kind] == 4) {
            const uint32_t w = __ldg(codes + lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t p = __ldg(pairs + (w >> (8 * i) & 255));
                const float2 v = __half22float2(reinterpret_cast<const __half2&>(p));
                x[2 * i] = __fmul_rn(v.x, norm);
                x[2 * i + 1] = __fmul_rn(v.y, norm);
            }
        } else {
            const uint2 w = __ldg(reinterpret_cast<const uint2*>(codes) + lane);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const uint32_t p = __ldg(pairs + ((i < 4 ? w.x : w.y) >> (8 * (i & 3)) & 255));
                x[i] = __fmul_rn(__low2float(reinterpret_cast<const __half2&>(p)), norm);
            }
        }
    }
    const CacheRows& out = a.rows[kind];
    store8(x, static_cast<T*>(out.data) + token * out.token_stride + head * out.head_stride, d, a.shape.dim, out.wide);
}

template <template <typename, int> class K, typename Args>
cudaError_t by_type_and_size(const Args& a, int type, cudaStream_t s)
{
    const int lanes = a.shape.padded / kEach;
    const int64_t threads = a.tokens * 2 * a.shape.heads * lanes;
    const int64_t blocks = (threads + kRowThreads - 1) / kRowThreads;
    if (blocks == 0) return cudaSuccess;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (lanes == 8) return K<T, 8>::launch(a, (unsigned)blocks, s);
        if (lanes == 16) return K<T, 16>::launch(a, (unsigned)blocks, s);
        return K<T, 32>::launch(a, (unsigned)blocks, s);
    };
    return type == LQ_F32 ? go(float()) : type == LQ_F16 ? go(__half()) : go(__nv_bfloat16());
}

template <typename T, int kLanes>
struct Write {
    static cudaError_t launch(const CacheWriteArgs& a, unsigned blocks, cudaStream_t s)
    {
        cache_write_kernel<T, kLanes><<<blocks, kRowThreads, 0, s>>>(a);
        return cudaGetLastError();
    }
};

template <typename T, int kLanes>
struct Read {
    static cudaError_t launch(const CacheReadArgs& a, unsigned blocks, cudaStream_t s)
    {
        cache_read_kernel<T, kLanes><<<blocks, kRowThreads, 0, s>>>(a);
        return cudaGetLastError();
    }
};

}  // namespace

cudaError_t launch_cache_write(const CacheWriteArgs& a, cudaStream_t s) { return by_type_and_size<Write>(a, a.rows[0].type, s); }
cudaError_t launch_cache_read(const CacheReadArgs& a, cudaStream_t s) { return by_type_and_size<Read>(a, a.rows[0].type, s); }

}  // namespace lq
