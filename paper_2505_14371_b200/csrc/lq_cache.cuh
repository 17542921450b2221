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
    const int32_t* table;               // [batch][table_width] page numbers; [batch * heads][table_width] where every head has its own
    const int32_t* lengths;
    float* lse;                         // [batch][heads * group] or NULL
    float* partial;                     // workspace, see lq_cache_attend.cuh; NULL: no sequence can be split
    uint32_t* flags;
    const int32_t* before;              // NULL, or how many tokens stand before each sequence's own: its last position is so much higher
    float* sums;                        // NULL, or [batch][heads * group] parts (cache_part_floats) that take the place of out and lse
    int64_t num_pages, table_width, window, before_most;        // before_most: tokens that *before can mean
    float scale;                        // of the scores, times log2(e)
    int32_t batch, group, group_blocks; // rows of the table; queries a head, and their blocks of 8
    int32_t row_heads, sequence_rows;   // heads that a row of the table serves: all, or 1; rows of a sequence: 1, or as many as there are heads
    CacheRowsOf by_rows;
    int32_t sms;                        // CTAs
};

// A prefix that all sequences of a batch share (lq_cache_shared.cu), and how what it and the sequences' own tokens give is joined.
struct CacheSharedArgs {
    CacheShape shape;
    const CacheTable* tables;
    CacheRows queries, out;
    CacheRotary rotary;
    const uint32_t* pages;
    const int32_t* prefix;              // [prefix_width] page numbers
    const int32_t* prefix_length;       // dev [1]
    const int32_t* lengths;             // dev [batch]: the sequences' own tokens
    float* lse;
    char* rows;                         // the queries as the matrix unit reads them, cache_shared_block_bytes a block of 128 rows (lq_cache_shared.cu)
    float* parts;                       // [splits * slots][batch][heads * group] parts of the prefix (cache_part_floats)
    float* own;                         // [batch][heads * group] parts of the sequences' own tokens
    uint32_t* flags;
    int64_t num_pages, prefix_most, own_most;   // the latter: tokens that the lengths can mean
    float scale;
    int32_t batch, group, splits;
    int32_t rests, slots, pairs, sms;   // what the queries' rounding leaves (cache_shared_rests), see cache_shared_slots, cache_shared_pairs
    int64_t wait_cycles;                // how long a wait may take
};

// Which pages a sequence's queries look at (lq_cache_choose.cu).
struct CacheBoundsArgs {
    CacheShape shape;
    const CacheTable* tables;
    const uint32_t* pages;
    const int32_t* which;               // [count] page numbers
    uint32_t* bounds;
    uint32_t* flags;
    int64_t num_pages, count;
    int32_t sms;
};
struct CacheChooseArgs {
    CacheShape shape;
    CacheRows queries;
    CacheRotary rotary;
    const uint32_t* bounds;
    const int32_t* table;
    const int32_t* lengths;
    int32_t* chosen;                    // [batch][heads][keep]
    int32_t* seen;                      // [batch][heads]
    uint32_t* scores;                   // [batch][heads][table_width]
    uint32_t* flags;
    int64_t num_pages, table_width;
    int32_t batch, group, first, last, keep, sms;
};
// Words of a page's bounds: for each head `padded` upper and `padded` lower bounds of a byte, then a scale a head, to a multiple of 16 bytes.
__host__ __device__ constexpr int cache_bounds_words(int heads, int padded) { return (heads * (padded / 2 + 1) + 3) / 4 * 4; }

cudaError_t launch_cache_write(const CacheWriteArgs& a, cudaStream_t s);
cudaError_t launch_cache_read(const CacheReadArgs& a, cudaStream_t s);
cudaError_t launch_cache_clear(uint32_t* flags, uint32_t seen);        // on the default stream

// One of each per padded head size (lq_cache_attend_<size>.cu).
cudaError_t launch_cache_attend_64(const CacheAttendArgs& a, cudaStream_t s);
cudaError_t launch_cache_attend_128(const CacheAttendArgs& a, cudaStream_t s);
cudaError_t launch_cache_attend_256(const CacheAttendArgs& a, cudaStream_t s);
cudaError_t launch_cache_bounds(const CacheBoundsArgs& a, cudaStream_t s);
cudaError_t launch_cache_choose(const CacheChooseArgs& a, cudaStream_t s);
cudaError_t launch_cache_shared_rows(const CacheSharedArgs& a, cudaStream_t s);
cudaError_t launch_cache_shared_prefix(const CacheSharedArgs& a, cudaStream_t s);
cudaError_t launch_cache_shared_join(const CacheSharedArgs& a, cudaStream_t s);
constexpr int64_t kCacheMostWait = (int64_t)1 << 32;     // clock cycles: some two seconds
// Into how many parts the prefix's tokens are split, and how many parts a query may leave of each (scores and sums of 128 rows that
// tensor memory holds at a time; `two`: weights are sums of two fp16 numbers, `rests`: see there).
int cache_shared_splits(int heads, bool pairs, int64_t rows, int64_t prefix_tokens, int type, int sms);
// What queries' rounding leaves: nothing, numbers beside the scores and weights, or (rows of 128 with weights of 11 bits, where tensor memory has
// no room for them and a second block's scores) numbers beside scores that give way to their weights.  In place a CTA has two blocks of rows and decodes for both,
// but a slot's next scores wait for its sums: that pays from four blocks on, if none is left alone.  8 heads, 4 queries each, sequences of 100 tokens of their
// own, prefixes of 2048, 16384 and 32768, us beside | in place: one block (4096 instead of 2048) 42, 56, 75 | 43, 59, 79; two 41, 75, 112 | 41, 78, 114;
// three 50, 99, 158 | 55, 119, 191; four 58, 130, 212 | 60, 123, 195; five 68, 162, 260 | 71, 165, 274; six 74, 171, 284 | 77, 172, 281; eight 95, 234, 410 | 91, 233, 375.
constexpr int kRestsBeside = 1, kRestsInPlace = 2;
__host__ __device__ constexpr int cache_shared_rests(int padded, bool two, int64_t rows)
{
    const int64_t blocks = (rows + 127) / 128;
    return padded == 128 && !two && blocks >= 4 && blocks % 2 == 0 ? kRestsInPlace : kRestsBeside;
}
__host__ __device__ constexpr int cache_shared_slots(int padded, bool two, int rests) { return padded == 256 || (padded == 128 && two && rests) ? 1 : 2; }
// Whether a CTA takes two blocks of rows where there are two.
__host__ __device__ constexpr bool cache_shared_pairs(int padded, bool two, int rests)
{
    return cache_shared_slots(padded, two, rests) == 2 && !(padded == 128 && rests == kRestsBeside);
}
// Workspace for a head's block of 128 rows: fp16 numbers, what their rounding left, a factor for each row.
__host__ __device__ constexpr int cache_shared_block_bytes(int padded) { return 128 * (4 * padded + 4); }
// Teams of 8 warps that share an SM in the attention kernel (its registers: rows of 256 need twice as many a thread), and what
// each may leave in the workspace: a record, then two partial sums of 8 queries.
__host__ __device__ constexpr int cache_attend_teams(int padded) { return padded == 256 ? 1 : 2; }
// Tiles of 16 tokens that a warp takes at a time, and those of a unit of work: two where two stages of two fit for every warp (rows of 128
// in 4 bits: one sequence of 130 001 tokens 47.0 us with one, 45.4 with two, of 200 tokens 8.8 and 6.3).
__host__ __device__ constexpr int cache_attend_pair(int padded, int bits_k, int bits_v) { return padded * (bits_k + bits_v) <= 1024 ? 2 : 1; }
__host__ __device__ constexpr int cache_attend_unit(int padded, int bits_k, int bits_v) { return 8 * cache_attend_pair(padded, bits_k, bits_v); }
constexpr int kCacheChooseKeys = 12288; // scores that a choosing CTA keeps in its shared memory; more are kept in the workspace
constexpr int kCacheRecordBytes = 16;
// What is left of one query over some of its tokens: sums of `padded` weighted values; reference of the scores, scale of the weights (both as
// base-2 exponents), denominator, unused.
__host__ __device__ constexpr int cache_part_floats(int padded) { return padded + 4; }
constexpr int cache_partial_floats(int padded) { return 8 * cache_part_floats(padded); }

}  // namespace lq
