// Host side of the quantised key-value cache: the object, the checks of its calls' arguments, and which kernels they launch.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "lq_cache.cuh"
#include "lq_internal.cuh"

using namespace lq;

struct lq_cache {
    CacheShape shape{};
    int32_t layers = 0, bits[2] = {0, 0}, device = 0, sms = 0;
    uint64_t seed = 0;
    CacheTable* tables = nullptr;          // dev [layers][2]
    uint32_t* flags = nullptr;             // dev [1]
    std::vector<float> levels;             // [layers][2][kCacheLevels], as rounded
};

namespace {

#define LQ_CUDA(expr)                                                                                      \
    do {                                                                                                   \
        const cudaError_t e_ = (expr);                                                                     \
        if (e_ != cudaSuccess)                                                                             \
            return lq_set_error(e_ == cudaErrorMemoryAllocation ? LQ_ENOMEM : LQ_ECUDA, "%s: %s", #expr,   \
                                cudaGetErrorString(e_));                                                   \
    } while (0)

// Makes the cache's device current for a call.
class OnDevice {
public:
    explicit OnDevice(int device) : error_(cudaGetDevice(&before_))
    {
        if (error_ == cudaSuccess && before_ != device) { error_ = cudaSetDevice(device); changed_ = error_ == cudaSuccess; }
    }
    ~OnDevice() { if (changed_) cudaSetDevice(before_); }
    cudaError_t error() const { return error_; }
private:
    int before_ = 0;
    bool changed_ = false;
    cudaError_t error_;
};

#define LQ_ON_DEVICE(cache)            \
    const OnDevice on_(cache->device); \
    LQ_CUDA(on_.error())

// Rounds a level set to numbers of 11 bits; false if it is not a set from 0 to 1 that increases, before and after.
bool rounded_levels(const float* levels, int n, float* out)
{
    if (levels[0] != 0.0f || levels[n - 1] != 1.0f) return false;
    for (int j = 0; j < n; ++j) {
        if (!(levels[j] >= 0.0f && levels[j] <= 1.0f)) return false;
        out[j] = __half2float(__float2half_rn(levels[j]));
        if (j > 0 && !(out[j] > out[j - 1])) return false;
    }
    return true;
}

void fill_search(CacheSearch& s, const float* levels, int n, bool nearest)
{
    const int edges = nearest ? n - 1 : n - 2;
    for (float& e : s.edge) e = INFINITY;
    for (int j = 1; j <= edges; ++j) {
        if (nearest) {
            const double middle = ((double)levels[j - 1] + (double)levels[j]) / 2;      // exact: multiples of 2^-25 up to 1
            float e = (float)middle;
            if (!((double)e > middle)) e = std::nextafterf(e, 2.0f);
            s.edge[j] = e;
        } else {
            s.edge[j] = levels[j];
        }
    }
    s.steps = 0;
    int at = 0, to = 0;                 // edges at or below the two ends of a bin (either end's number may be in it)
    for (int b = 0; b <= kCacheBins; ++b) {
        while (at < edges && (double)s.edge[at + 1] <= (b - 0.5) / kCacheBins) ++at;
        while (to < edges && (double)s.edge[to + 1] <= (b + 0.5) / kCacheBins) ++to;
        s.start[b] = (uint8_t)at;
        s.steps = std::max(s.steps, to - at);
    }
    // the coarsest bins of the pattern that part all edges; the first one has to start below the first edge
    auto bits = [](float v) { uint32_t b; std::memcpy(&b, &v, sizeof b); return b; };
    s.entries = 0;
    for (int shift = 19; shift >= 15 && !s.entries; --shift) {
        const uint32_t first = (bits(s.edge[1]) - 1) >> shift, last = bits(1.0f) >> shift;
        if (last - first >= (uint32_t)kCacheBins) break;
        bool parted = true;
        for (int j = 2; j <= edges; ++j) parted = parted && bits(s.edge[j]) >> shift != bits(s.edge[j - 1]) >> shift;
        if (!parted) continue;
        int j = 0;                      // edges in the bins before
        for (uint32_t b = first; b <= last; ++b) {
            uint32_t e = ((uint32_t)j << shift) - (b << shift);
            if (j < edges && bits(s.edge[j + 1]) >> shift == b) {
                e += (1u << shift) - (bits(s.edge[j + 1]) & ((1u << shift) - 1));       // a number at or past the edge carries
                ++j;
            }
            s.entry[b - first] = e;
        }
        const uint32_t low = first << shift;
        std::memcpy(&s.lowest, &low, sizeof low);
        s.shift = shift; s.first = (int32_t)first; s.entries = (int32_t)(last - first + 1);
    }
}

void fill_table(CacheTable& t, const float* levels, int bits)
{
    std::memset(&t, 0, sizeof t);
    for (int j = 0; j < 1 << bits; ++j) t.levels[j] = levels[j];
    fill_search(t.nearest, levels, 1 << bits, true);
    fill_search(t.floor, levels, 1 << bits, false);
    auto half_of = [&](uint32_t sym) {
        const __half_raw h = __float2half_rn(levels[sym >> 1]);
        return (uint32_t)h.x | ((sym & 1) << 15);
    };
    for (uint32_t b = 0; b < kCachePairs; ++b)
        t.pairs[b] = bits == 3 ? half_of(b & 15) | half_of(b >> 4) << 16 : half_of(b) | half_of(b) << 16;
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int type_size(int type) { return type == LQ_F32 ? 4 : 2; }

// Checks one row argument and brings it into the kernels' form; `n`: rows of tokens.
int take_rows(const char* name, const lq_rows* r, int64_t n, int heads, bool output, CacheRows* out)
{
    if (!r) return lq_set_error(LQ_EINVAL, "%s is NULL", name);
    if (r->type != LQ_F32 && r->type != LQ_F16 && r->type != LQ_BF16) return lq_set_error(LQ_EINVAL, "%s: type %d is not one of LQ_F32, LQ_F16, LQ_BF16", name, r->type);
    if (n > 0 && !r->data) return lq_set_error(LQ_EINVAL, "%s: data is NULL", name);
    const int size = type_size(r->type);
    if (!aligned(r->data, (size_t)size)) return lq_set_error(LQ_EINVAL, "%s must be %d-byte aligned", name, size);
    if (output && ((n > 1 && r->token_stride == 0) || (heads > 1 && r->head_stride == 0)))
        return lq_set_error(LQ_EINVAL, "%s: rows of an output share memory (a stride is 0)", name);
    out->data = r->data;
    const int64_t token = n > 1 ? r->token_stride : 0, head = heads > 1 ? r->head_stride : 0;
    for (const int64_t s : {token, head})
        if (s > INT32_MAX / size || s < -(INT32_MAX / size)) return lq_set_error(LQ_EINVAL, "%s: a stride is 2^31 bytes or more", name);
    out->token_bytes = (int32_t)token * size;
    out->head_bytes = (int32_t)head * size;
    out->type = r->type;
    out->wide = aligned(r->data, 16) && out->token_bytes % 16 == 0 && out->head_bytes % 16 == 0;
    return LQ_OK;
}

int take_rotary(const lq_rotary* r, const CacheShape& shape, bool need_at, CacheRotary* out)
{
    std::memset(out, 0, sizeof *out);
    if (!r) return LQ_OK;
    if (!r->table || !aligned(r->table, 4)) return lq_set_error(LQ_EINVAL, "rotary table is NULL or not 4-byte aligned");
    if (r->dim < 2 || r->dim % 2 || r->dim > shape.dim)
        return lq_set_error(LQ_EINVAL, "rotary dim %d is not an even number from 2 to head_dim = %d", r->dim, shape.dim);
    if (r->positions < 1 || r->positions > INT32_MAX) return lq_set_error(LQ_EINVAL, "rotary table has %lld positions: 1 to 2^31 - 1 are wanted", (long long)r->positions);
    if (need_at && !r->at) return lq_set_error(LQ_EINVAL, "rotary positions (at) are NULL");
    if (!aligned(r->at, 8)) return lq_set_error(LQ_EINVAL, "rotary positions (at) must be 8-byte aligned");
    out->table = r->table; out->at = r->at; out->positions = r->positions; out->dim = r->dim; out->interleaved = r->interleaved != 0;
    out->wide = r->dim % 16 == 0 && aligned(r->table, 16);
    return LQ_OK;
}

int check_pages(const lq_cache* c, int32_t layer, const void* pages, int64_t num_pages)
{
    if (layer < 0 || layer >= c->layers) return lq_set_error(LQ_EINVAL, "layer %d out of range", layer);
    if (num_pages < 0 || num_pages > INT32_MAX || (num_pages << c->shape.page_shift) > (int64_t)1 << 32)
        return lq_set_error(LQ_EINVAL, "num_pages = %lld: a layer has at most 2^31 - 1 pages and 2^32 slots", (long long)num_pages);
    if (num_pages > 0 && !pages) return lq_set_error(LQ_EINVAL, "pages is NULL");
    if (!aligned(pages, 16)) return lq_set_error(LQ_EINVAL, "pages must be 16-byte aligned");
    return LQ_OK;
}

int check_slots(const lq_cache* c, int64_t tokens, const int64_t* slots)
{
    const int64_t most = INT32_MAX / c->shape.heads;        // (token, head) pairs are counted in 31 bits
    if (tokens < 0 || tokens > most) return lq_set_error(LQ_EINVAL, "tokens = %lld out of [0, %lld]", (long long)tokens, (long long)most);
    if (tokens > 0 && !slots) return lq_set_error(LQ_EINVAL, "slots is NULL");
    if (!aligned(slots, 8)) return lq_set_error(LQ_EINVAL, "slots must be 8-byte aligned");
    return LQ_OK;
}

// r / heads = floor(r * ceil(2^(31 + s) / heads) / 2^(31 + s)) for r < 2^31 with 2^s >= heads.
CacheRowsOf rows_of(int heads)
{
    CacheRowsOf d{};
    while ((1 << d.shift) < heads) ++d.shift;
    d.factor = (uint32_t)((((uint64_t)1 << (31 + d.shift)) + heads - 1) / heads);
    return d;
}

// Most tiles of 16 tokens that a sequence has to be read of.
int64_t tiles_of(const lq_cache* c, int64_t table_width, int64_t window)
{
    const int64_t all = (table_width << c->shape.page_shift) / 16;
    return window > 0 ? std::min<int64_t>(all, window / 16 + 2) : all;
}

// None where no sequence can be split: a unit never is.
int64_t workspace_of(const lq_cache* c, int64_t table_width, int64_t window)
{
    const CacheShape& s = c->shape;
    if (tiles_of(c, table_width, window) <= cache_attend_unit(s.padded, s.sym_bits[0], s.sym_bits[1])) return 0;
    return (int64_t)c->sms * cache_attend_teams(s.padded) * (kCacheRecordBytes + 2 * 4 * cache_partial_floats(s.padded));
}

#define LQ_TRY(expr) do { const int c_ = (expr); if (c_ != LQ_OK) return c_; } while (0)

}  // namespace

extern "C" {

int lq_cache_create(lq_cache** out, int32_t num_layers, int32_t kv_heads, int32_t head_dim, int32_t page_size, int32_t bits_keys,
                    int32_t bits_values, int32_t q, uint64_t seed)
{
    if (!out) return lq_set_error(LQ_EINVAL, "out is NULL");
    *out = nullptr;
    if (num_layers < 1 || num_layers > 4096) return lq_set_error(LQ_EINVAL, "num_layers must be in [1, 4096], got %d", num_layers);
    if (kv_heads < 1 || kv_heads > 1024) return lq_set_error(LQ_EINVAL, "kv_heads must be in [1, 1024], got %d", kv_heads);
    if (head_dim < 1 || head_dim > 256) return lq_set_error(LQ_EINVAL, "head_dim must be in [1, 256], got %d", head_dim);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)))
        return lq_set_error(LQ_EINVAL, "page_size must be a power of two from 16 to 1024, got %d", page_size);
    for (const int b : {bits_keys, bits_values})
        if (b != 3 && b != 7) return lq_set_error(LQ_EINVAL, "bits must be 3 or 7 (symbols of 4 or 8 bits), got %d", b);
    if (q < 0 || q > 2) return lq_set_error(LQ_EINVAL, "q must be 0 (infinity norm), 1 or 2, got %d", q);

    lq_cache* c = new (std::nothrow) lq_cache;
    if (!c) return lq_set_error(LQ_ENOMEM, "host allocation failed");
    CacheShape& s = c->shape;
    s.heads = kv_heads; s.dim = head_dim; s.padded = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; s.q = q;
    while ((1 << s.page_shift) < page_size) ++s.page_shift;
    c->layers = num_layers; c->seed = seed;
    c->bits[0] = bits_keys; c->bits[1] = bits_values;
    for (int k = 0; k < 2; ++k) { s.sym_bits[k] = c->bits[k] + 1; s.row_words[k] = s.padded * s.sym_bits[k] / 32; }
    s.head_words = page_size * (s.row_words[0] + s.row_words[1] + 2);
    s.page_words = s.head_words * kv_heads;

    std::vector<CacheTable> host;
    try {
        c->levels.resize((size_t)num_layers * 2 * kCacheLevels);
        host.resize((size_t)num_layers * 2);
    } catch (const std::bad_alloc&) {
        delete c;
        return lq_set_error(LQ_ENOMEM, "host allocation failed");
    }
    for (int k = 0; k < 2; ++k) {
        float uniform[kCacheLevels];
        const int n = 1 << c->bits[k];
        for (int j = 0; j < n; ++j) uniform[j] = (float)((double)j / (double)(n - 1));
        CacheTable t;
        rounded_levels(uniform, n, uniform);
        fill_table(t, uniform, c->bits[k]);
        for (int m = 0; m < num_layers; ++m) {
            host[(size_t)m * 2 + k] = t;
            std::memcpy(&c->levels[((size_t)m * 2 + k) * kCacheLevels], t.levels, sizeof t.levels);
        }
    }
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, c->device);
    // the attention kernel places its shared memory by address (lq_cache_attend.cuh)
    int reserved = 0;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&reserved, cudaDevAttrReservedSharedMemoryPerBlock, c->device);
    if (e == cudaSuccess && reserved > 1024) {
        delete c;
        return lq_set_error(LQ_ECUDA, "cache setup: %d bytes of shared memory are the system's, 1024 at most are expected", reserved);
    }
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&c->tables), host.size() * sizeof(CacheTable));
    if (e == cudaSuccess) e = cudaMemcpy(c->tables, host.data(), host.size() * sizeof(CacheTable), cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&c->flags), sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMemset(c->flags, 0, sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        cudaFree(c->tables); cudaFree(c->flags);
        delete c;
        return lq_set_error(e == cudaErrorMemoryAllocation ? LQ_ENOMEM : LQ_ECUDA, "cache setup: %s", cudaGetErrorString(e));
    }
    *out = c;
    return LQ_OK;
}

int lq_cache_destroy(lq_cache* cache)
{
    if (!cache) return LQ_OK;
    {
        const OnDevice on(cache->device);
        cudaDeviceSynchronize();
        cudaFree(cache->tables); cudaFree(cache->flags);
    }
    delete cache;
    return LQ_OK;
}

int64_t lq_cache_page_words(const lq_cache* cache) { return cache ? (int64_t)cache->shape.page_words : (int64_t)lq_set_error(LQ_EINVAL, "cache is NULL"); }

int64_t lq_cache_workspace(const lq_cache* cache, int64_t table_width, int64_t window)
{
    if (!cache) return lq_set_error(LQ_EINVAL, "cache is NULL");
    if (table_width < 0 || table_width > INT32_MAX || window < 0) return lq_set_error(LQ_EINVAL, "table_width or window out of range");
    return workspace_of(cache, table_width, window);
}

int lq_cache_info(const lq_cache* cache, int32_t* kv_heads, int32_t* head_dim, int32_t* page_size, int32_t* device)
{
    if (!cache) return lq_set_error(LQ_EINVAL, "cache is NULL");
    if (kv_heads) *kv_heads = cache->shape.heads;
    if (head_dim) *head_dim = cache->shape.dim;
    if (page_size) *page_size = 1 << cache->shape.page_shift;
    if (device) *device = cache->device;
    return LQ_OK;
}

int lq_cache_set_levels(lq_cache* cache, int32_t layer, int32_t kind, const float* host_levels, int32_t n)
{
    if (!cache || !host_levels) return lq_set_error(LQ_EINVAL, "NULL argument");
    if (layer < 0 || layer >= cache->layers) return lq_set_error(LQ_EINVAL, "layer %d out of range", layer);
    if (kind != LQ_KEYS && kind != LQ_VALUES) return lq_set_error(LQ_EINVAL, "kind %d is neither LQ_KEYS nor LQ_VALUES", kind);
    if (n != 1 << cache->bits[kind]) return lq_set_error(LQ_EINVAL, "the set has %d levels, got %d", 1 << cache->bits[kind], n);
    CacheTable t;
    float rounded[kCacheLevels] = {};
    if (!rounded_levels(host_levels, n, rounded))
        return lq_set_error(LQ_EINVAL, "levels must start at 0, end at 1 and increase, also as numbers of 11 bits");
    fill_table(t, rounded, cache->bits[kind]);
    LQ_ON_DEVICE(cache);
    LQ_CUDA(cudaDeviceSynchronize());
    LQ_CUDA(cudaMemcpy(cache->tables + (size_t)layer * 2 + kind, &t, sizeof t, cudaMemcpyHostToDevice));
    LQ_CUDA(cudaDeviceSynchronize());
    std::memcpy(&cache->levels[((size_t)layer * 2 + kind) * kCacheLevels], rounded, sizeof rounded);
    return LQ_OK;
}

int lq_cache_get_levels(const lq_cache* cache, int32_t layer, int32_t kind, float* host_levels, int32_t n)
{
    if (!cache || !host_levels) return lq_set_error(LQ_EINVAL, "NULL argument");
    if (layer < 0 || layer >= cache->layers) return lq_set_error(LQ_EINVAL, "layer %d out of range", layer);
    if (kind != LQ_KEYS && kind != LQ_VALUES) return lq_set_error(LQ_EINVAL, "kind %d is neither LQ_KEYS nor LQ_VALUES", kind);
    if (n != 1 << cache->bits[kind]) return lq_set_error(LQ_EINVAL, "the set has %d levels, got %d", 1 << cache->bits[kind], n);
    std::memcpy(host_levels, &cache->levels[((size_t)layer * 2 + kind) * kCacheLevels], (size_t)n * sizeof(float));
    return LQ_OK;
}

int lq_cache_status(lq_cache* cache, uint32_t* flags)
{
    if (!cache || !flags) return lq_set_error(LQ_EINVAL, "NULL argument");
    LQ_ON_DEVICE(cache);
    LQ_CUDA(cudaDeviceSynchronize());
    LQ_CUDA(cudaMemcpy(flags, cache->flags, sizeof *flags, cudaMemcpyDeviceToHost));
    if (*flags) LQ_CUDA(launch_cache_clear(cache->flags, *flags));      // what another thread's call sets meanwhile stays
    LQ_CUDA(cudaDeviceSynchronize());
    return LQ_OK;
}

int lq_cache_write(lq_cache* cache, int32_t layer, const lq_rows* keys, const lq_rows* values, int64_t tokens, const int64_t* slots,
                   uint32_t* pages, int64_t num_pages, int64_t step, const lq_rotary* rotary, void* stream)
{
    if (!cache) return lq_set_error(LQ_EINVAL, "cache is NULL");
    CacheWriteArgs a{};
    LQ_TRY(check_pages(cache, layer, pages, num_pages));
    LQ_TRY(check_slots(cache, tokens, slots));
    LQ_TRY(take_rows("keys", keys, tokens, cache->shape.heads, false, &a.rows[0]));
    LQ_TRY(take_rows("values", values, tokens, cache->shape.heads, false, &a.rows[1]));
    if (keys->type != values->type) return lq_set_error(LQ_EINVAL, "keys and values have to be of one type");
    LQ_TRY(take_rotary(rotary, cache->shape, tokens > 0, &a.rotary));
    if (step < -1 || step > (int64_t)UINT32_MAX) return lq_set_error(LQ_EINVAL, "step = %lld is neither -1 nor in [0, 2^32)", (long long)step);
    if (tokens == 0) return LQ_OK;
    a.shape = cache->shape; a.tables = cache->tables + (size_t)layer * 2;
    a.slots = slots; a.pages = pages; a.flags = cache->flags; a.tokens = tokens; a.num_slots = num_pages << cache->shape.page_shift;
    a.by_head = rows_of(cache->shape.heads);
    a.seed_lo = (uint32_t)cache->seed; a.seed_hi = (uint32_t)(cache->seed >> 32);
    a.layer = (uint32_t)layer; a.unbiased = step >= 0; a.step = step >= 0 ? (uint32_t)step : 0;
    LQ_ON_DEVICE(cache);
    LQ_CUDA(launch_cache_write(a, (cudaStream_t)stream));
    return LQ_OK;
}

int lq_cache_read(lq_cache* cache, int32_t layer, const uint32_t* pages, int64_t num_pages, int64_t tokens, const int64_t* slots,
                  const lq_rows* keys, const lq_rows* values, void* stream)
{
    if (!cache) return lq_set_error(LQ_EINVAL, "cache is NULL");
    CacheReadArgs a{};
    LQ_TRY(check_pages(cache, layer, pages, num_pages));
    LQ_TRY(check_slots(cache, tokens, slots));
    LQ_TRY(take_rows("keys", keys, tokens, cache->shape.heads, true, &a.rows[0]));
    LQ_TRY(take_rows("values", values, tokens, cache->shape.heads, true, &a.rows[1]));
    if (keys->type != values->type) return lq_set_error(LQ_EINVAL, "keys and values have to be of one type");
    if (tokens == 0) return LQ_OK;
    a.shape = cache->shape; a.tables = cache->tables + (size_t)layer * 2;
    a.slots = slots; a.pages = pages; a.flags = cache->flags; a.tokens = tokens; a.num_slots = num_pages << cache->shape.page_shift;
    a.by_head = rows_of(cache->shape.heads);
    LQ_ON_DEVICE(cache);
    LQ_CUDA(launch_cache_read(a, (cudaStream_t)stream));
    return LQ_OK;
}

int lq_cache_attend(lq_cache* cache, int32_t layer, const lq_rows* queries, int64_t batch, int32_t heads, const uint32_t* pages,
                    int64_t num_pages, const int32_t* table, int64_t table_width, const int32_t* lengths, float scale, int64_t window,
                    const lq_rotary* rotary, const lq_rows* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (!cache) return lq_set_error(LQ_EINVAL, "cache is NULL");
    const CacheShape& s = cache->shape;
    CacheAttendArgs a{};
    LQ_TRY(check_pages(cache, layer, pages, num_pages));
    if (batch < 0 || batch > 1 << 24) return lq_set_error(LQ_EINVAL, "batch = %lld out of [0, 2^24]", (long long)batch);
    if (heads < s.heads || heads % s.heads || heads > 1 << 16)
        return lq_set_error(LQ_EINVAL, "query heads (%d) have to be a multiple of the cache's %d, at most 65536", heads, s.heads);
    LQ_TRY(take_rows("queries", queries, batch, heads, false, &a.queries));
    LQ_TRY(take_rows("out", out, batch, heads, true, &a.out));
    if (queries->type != out->type) return lq_set_error(LQ_EINVAL, "queries and out have to be of one type");
    if (table_width < 0 || table_width > INT32_MAX) return lq_set_error(LQ_EINVAL, "table_width = %lld out of range", (long long)table_width);
    if (batch > 0 && (!lengths || (table_width > 0 && !table))) return lq_set_error(LQ_EINVAL, "table or lengths is NULL");
    if (!aligned(table, 4) || !aligned(lengths, 4) || !aligned(lse, 4)) return lq_set_error(LQ_EINVAL, "table, lengths and lse must be 4-byte aligned");
    a.scale = scale * 1.44269504088896341f;
    if (!std::isfinite(a.scale)) return lq_set_error(LQ_EINVAL, "scale is not a finite number (or above 2^127, where its base-2 form is none)");
    if (window < 0) return lq_set_error(LQ_EINVAL, "window = %lld is negative", (long long)window);
    LQ_TRY(take_rotary(rotary, s, false, &a.rotary));
    const int64_t needed = workspace_of(cache, table_width, window);
    if (needed > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < needed))
        return lq_set_error(LQ_EINVAL, "workspace has to be 16-byte aligned and of %lld bytes or more", (long long)needed);
    a.group = heads / s.heads; a.group_blocks = (a.group + 7) / 8;
    // the dealing out of work multiplies its units with the grid in 64 bits
    const double tokens = (double)std::min<int64_t>(table_width << s.page_shift, INT32_MAX);
    if ((tokens / 128 + 1) * (double)batch * s.heads * a.group_blocks * cache->sms * 2 > 4e18)
        return lq_set_error(LQ_EINVAL, "batch, heads and table_width are too large together");
    if (batch == 0) return LQ_OK;
    a.shape = s; a.tables = cache->tables + (size_t)layer * 2;
    a.pages = pages; a.table = table; a.lengths = lengths; a.lse = lse; a.partial = needed > 0 ? static_cast<float*>(workspace) : nullptr; a.flags = cache->flags;
    a.num_pages = num_pages; a.table_width = table_width; a.window = window;
    a.batch = (int32_t)batch;
    a.sms = cache->sms;
    LQ_ON_DEVICE(cache);
    LQ_CUDA(s.padded == 64 ? launch_cache_attend_64(a, (cudaStream_t)stream)
            : s.padded == 128 ? launch_cache_attend_128(a, (cudaStream_t)stream) : launch_cache_attend_256(a, (cudaStream_t)stream));
    return LQ_OK;
}

}  // extern "C"
