// The quantised key-value cache: what its host side and its kernels share (not part of the public ABI).
//
// Layout of a page, in 32-bit words, for each head in turn (RowShape::head_words of them):
//   page_size rows of keys, page_size rows of values, page_size norms of keys, page_size norms of values (fp32).
// A row holds `padded` symbols of 4 or 8 bits, little endian, 2 * level index + sign, zeros past head_dim.  padded is 64,
// 128 or 256, the sizes that the attention kernel is compiled for.  Rows stay in the order of their tokens and coordinates:
// a warp of the attention kernel reads 16 tokens, and with tokens and coordinates dealt to lanes as below
// each lane's share of a row is one run of 4 to 16 bytes, so no other arrangement is needed to feed matrix instructions.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "lq.h"

namespace lq {

constexpr int kCacheLevels = 128;       // most levels of a set (7 bits)
constexpr int kCachePairs = 256;        // entries of the look-up table by bytes

constexpr int kCacheBins = 2048;

// Where u falls: index = how many of edge[1..] are <= u.  For rounding to the nearest level edge[j] is the least fp32 number above
// the middle of levels j - 1 and j; for unbiased rounding it is level j, up to the last but one.  Entries behind are +infinity.
// Two searches, by one look-up where no bin of u's pattern (16 to 256 bins an octave, from the first edge's to 1) holds two edges, else by
// linear bins and steps (16384 tokens of 8 heads of 128 written, 4 bits: 42 us and 80; 9600 of 10 heads of 41, unbiased, 8 bits: 36 and 47).
struct alignas(16) CacheSearch {
    // 1: u's pattern is cut off `shift` bits; entry[bin - first] + pattern has the index above bit `shift`.  Numbers below `lowest`, the
    // first bin's start, are taken as it.  entries 0: no such table.
    int32_t shift, first, entries;
    float lowest;
    // 2: by round(2048 u): edges at or below all of the bin's numbers, and the most that are inside one
    int32_t steps, pad[3];
    float edge[kCacheLevels + 4];
    uint8_t start[kCacheBins + 16];
    uint32_t entry[kCacheBins];
};

// Device tables of one (layer, keys or values).
struct alignas(16) CacheTable {
    float levels[kCacheLevels];         // numbers of 11 bits (set_levels rounds them)
    CacheSearch nearest, floor;
    // By byte of a row: 4-bit symbols: the two signed levels as fp16, the first symbol's in the low half;
    // 8-bit symbols: the signed level as fp16 in both halves.
    uint32_t pairs[kCachePairs];
};

struct CacheShape {
    int32_t heads, dim, padded;
    int32_t page_shift;                 // log2(tokens of a page)
    int32_t sym_bits[2];                // 4 or 8: keys, values
    int32_t row_words[2];
    int32_t q;                          // norm: 0 infinity, 1, 2
    int32_t head_words, page_words;     // (at most 2^28)
};

// Rows [tokens][heads][dim] with any strides between tokens and heads, coordinates side by side.
struct CacheRows {
    void* data;
    int32_t token_bytes, head_bytes;    // strides
    int32_t type;                       // LQ_F32, LQ_F16, LQ_BF16
    int32_t wide;                       // every row starts on a 16-byte boundary
};

struct CacheRotary {
    const float* table;                 // [positions][dim]: cosines of dim / 2 angles, then sines; NULL: none
    const int64_t* at;                  // position of every token; NULL in lq_cache_attend: the last token's
    int64_t positions;
    int32_t dim;
    int32_t interleaved;
    int32_t wide;                       // 8 coordinates of a lane are turned alike, and their angles read 16 bytes at a time
};

// r / heads for 0 <= r < 2^31 as a product: umulhi(2 r, factor) >> shift.
struct CacheRowsOf { uint32_t factor, shift; };

struct CacheWriteArgs {
    CacheShape shape;
    const CacheTable* tables;           // keys, values
    CacheRows rows[2];
    CacheRotary rotary;
    const int64_t* slots;
    uint32_t* pages;
    uint32_t* flags;
    int64_t tokens, num_slots;
    CacheRowsOf by_head;
    uint32_t seed_lo, seed_hi, layer, step;
    int32_t unbiased;
};

struct CacheReadArgs {
    CacheShape shape;
    const CacheTable* tables;
    CacheRows rows[2];
    const int64_t* slots;
    const uint32_t* pages;
    uint32_t* flags;
    int64_t tokens, num_slots;
    CacheRowsOf by_head;
};

struct CacheAttendArgs {
    CacheShape shape;
    const CacheTable* tables;
    CacheRows queries, out;
    CacheRotary rotary;
    const uint32_t* pages;
    const int32_t* table;               // [batch][table_width] page numbers
    const int32_t* lengths;
    float* lse;                         // [batch][heads * group] or NULL
    float* partial;                     // workspace, see lq_cache_attend.cuh; NULL: no sequence can be split
    uint32_t* flags;
    int64_t num_pages, table_width, window;
    float scale;                        // of the scores, times log2(e)
    int32_t batch, group, group_blocks; // queries a head, and their blocks of 8
    int32_t sms;                        // CTAs
};

cudaError_t launch_cache_write(const CacheWriteArgs& a, cudaStream_t s);
cudaError_t launch_cache_read(const CacheReadArgs& a, cudaStream_t s);
cudaError_t launch_cache_clear(uint32_t* flags, uint32_t seen);        // on the default stream

// One of each per padded head size (lq_cache_attend_<size>.cu).
cudaError_t launch_cache_attend_64(const CacheAttendArgs& a, cudaStream_t s);
cudaError_t launch_cache_attend_128(const CacheAttendArgs& a, cudaStream_t s);
cudaError_t launch_cache_attend_256(const CacheAttendArgs& a, cudaStream_t s);
// Teams of 8 warps that share an SM in the attention kernel (its registers: rows of 256 need twice as many a thread), and what
// each may leave in the workspace: a record, then two partial sums of 8 queries.
__host__ __device__ constexpr int cache_attend_teams(int padded) { return padded == 256 ? 1 : 2; }
// Tiles of 16 tokens that a warp takes at a time, and those of a unit of work: two where two stages of two fit for every warp (rows of 128
// in 4 bits: one sequence of 130 001 tokens 47.0 us with one, 45.4 with two, of 200 tokens 8.8 and 6.3).
__host__ __device__ constexpr int cache_attend_pair(int padded, int bits_k, int bits_v) { return padded * (bits_k + bits_v) <= 1024 ? 2 : 1; }
__host__ __device__ constexpr int cache_attend_unit(int padded, int bits_k, int bits_v) { return 8 * cache_attend_pair(padded, bits_k, bits_v); }
constexpr int kCacheRecordBytes = 16;
constexpr int cache_partial_floats(int padded) { return 8 * (padded + 4); }

}  // namespace lq
