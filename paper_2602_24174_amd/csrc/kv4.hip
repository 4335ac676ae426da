// The 4-bit KV cache behind the C ABI: append, read, attention.  Layout and kernels: kernels_kv4.h.
#include "kernels_kv4.h"
#include <algorithm>
#include <mutex>

namespace {

// A kernel's largest dynamic LDS, set once per device where it is beyond the default
struct LdsRoom {
    std::mutex mu;
    bool ready[16] = {};
    tasc_status for_kernel(const void* kernel, int bytes) {
        if (bytes <= 65536) return TASC_OK;
        int dev = 0;
        TASC_HIP(hipGetDevice(&dev));
        std::lock_guard<std::mutex> lock(mu);
        if (ready[dev & 15]) return TASC_OK;
        TASC_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        ready[dev & 15] = true;
        return TASC_OK;
    }
};

template <int HD>
tasc_status attend_rows(const Kv4Attn& a, hipStream_t st) {
    const int64_t pairs = (int64_t)a.max_rows * (a.H / a.Hkv), per = 32 * kKv4RowWaves;
    const int lds = kv4_attention_rows_lds<HD>();
    static LdsRoom room;
    const tasc_status rc = room.for_kernel(reinterpret_cast<const void*>(&k_kv4_attention_rows<HD>), lds);
    if (rc != TASC_OK) return rc;
    k_kv4_attention_rows<HD><<<dim3((unsigned)((pairs + per - 1) / per * a.batch * a.Hkv)), dim3(64 * kKv4RowWaves), lds, st>>>(a);
    return TASC_OK;
}
template <int HD, int MT, int KW>
tasc_status attend(Kv4Attn a, hipStream_t st) {
    // four waves a workgroup (KW at least), fewer where the pairs end before
    const int64_t pairs = (int64_t)a.max_rows * (a.H / a.Hkv), waves = (pairs + 16 * MT - 1) / (16 * MT);
    constexpr int MOST = KW < 4 ? 4 / KW : 1;
    a.row_waves = (int)std::min<int64_t>(waves, MOST);
    const int64_t tiles = (waves + a.row_waves - 1) / a.row_waves;
    const int lds = kv4_attention_lds<HD, MT, KW>(a.row_waves * KW);
    static LdsRoom room;
    const tasc_status rc = room.for_kernel(reinterpret_cast<const void*>(&k_kv4_attention<HD, MT, KW>), kv4_attention_lds<HD, MT, KW>(MOST * KW));
    if (rc != TASC_OK) return rc;
    k_kv4_attention<HD, MT, KW><<<dim3((unsigned)(tiles * a.chunks), (unsigned)(a.batch * a.Hkv)), dim3((unsigned)(64 * a.row_waves * KW)), lds, st>>>(a);
    return TASC_OK;
}
template <int HD>
tasc_status attend_hd(const Kv4Attn& a, int kw, hipStream_t st) {
    const int64_t pairs = (int64_t)a.max_rows * (a.H / a.Hkv);
    tasc_status rc;
    if (kw == 8) rc = attend<HD, 1, 8>(a, st);
    else if (kw == 4) rc = attend<HD, 1, 4>(a, st);
    else if (kw == 1) rc = attend_rows<HD>(a, st);
    else if (pairs <= 16) rc = attend<HD, 1, 2>(a, st);
    else rc = attend<HD, 2, 2>(a, st);
    if (rc != TASC_OK) return rc;
    if (a.chunks > 8) k_kv4_merge<HD, true><<<dim3((unsigned)(a.max_rows * a.H), (unsigned)a.batch), dim3(256), 0, st>>>(a);
    else if (a.chunks > 1) k_kv4_merge<HD, false><<<dim3((unsigned)(a.max_rows * ((a.H + 1024 / HD - 1) / (1024 / HD))), (unsigned)a.batch), dim3(256), 0, st>>>(a);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

tasc_status check_cache(const char* who, const tasc_kv4_cache* c) {
    TASC_REQUIRE(c && c->pool, "%s: null cache", who);
    TASC_REQUIRE(kv4_head_dim_ok(c->head_dim), "%s: head_dim %d is none of 32, 64, 128", who, c->head_dim);
    TASC_REQUIRE(c->n_kv_heads >= 1 && c->n_kv_heads <= 1024, "%s: %d KV heads outside [1, 1024]", who, c->n_kv_heads);
    TASC_REQUIRE(c->n_pages >= 1 && c->n_pages < 1 << 27, "%s: %d pages outside [1, 2^27)", who, c->n_pages);
    TASC_REQUIRE(((uintptr_t)c->pool & 127) == 0, "%s: the pool must be 128-byte aligned", who);
    return TASC_OK;
}
// f(head_dim as a type)
template <typename F>
void with_hd(int hd, F f) {
    if (hd == 128) f(std::integral_constant<int, 128>{});
    else if (hd == 64) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 32>{});
}

constexpr int kMostChunks = 64;
constexpr int64_t kMostBlocks = 1 << 24;                    // workgroups of 256 threads: a launch has less than 2^32 threads a dimension

}  // namespace

tasc_status tasc_kv4_attend(Kv4Attn a, int hd, const Kv4Order& o, hipStream_t st) {
    a.chunks = o.chunks;
    a.chunk_tiles = o.chunk_tiles;
    return hd == 128 ? attend_hd<128>(a, o.kw, st) : hd == 64 ? attend_hd<64>(a, o.kw, st) : attend_hd<32>(a, o.kw, st);
}

extern "C" size_t tasc_kv4_page_bytes(int32_t n_kv_heads, int32_t head_dim) {
    if (!kv4_head_dim_ok(head_dim) || n_kv_heads < 1 || n_kv_heads > 1024) return 0;
    return (size_t)n_kv_heads * kv4_head_bytes(head_dim);
}

extern "C" tasc_status tasc_kv4_append(const tasc_kv4_cache* c, const void* k, const void* v, tasc_dtype dtype, int64_t k_stride, int64_t v_stride,
                                       const int32_t* slots, int32_t rows, void* stream) {
    tasc_status rc = check_cache("kv4_append", c);
    if (rc != TASC_OK) return rc;
    TASC_REQUIRE(rows >= 0, "kv4_append: %d rows", rows);
    if (rows == 0) return TASC_OK;
    TASC_REQUIRE(k && v && slots, "kv4_append: null argument");
    TASC_REQUIRE(dtype == TASC_F32 || dtype == TASC_BF16, "kv4_append: dtype %d", (int)dtype);
    const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
    TASC_REQUIRE(k_stride >= 0 && v_stride >= 0, "kv4_append: negative row stride");
    const int es = dtype == TASC_F32 ? 4 : 2;
    TASC_REQUIRE((uintptr_t)k % es == 0 && (uintptr_t)v % es == 0, "kv4_append: keys and values must be aligned to their type");
    const bool vec = (((uintptr_t)k | (uintptr_t)v | (uintptr_t)(k_stride * es) | (uintptr_t)(v_stride * es)) & 15) == 0;
    const Kv4Rows a{(uint8_t*)c->pool, c->n_pages, c->n_kv_heads, rows, slots};
    const int64_t blocks = ((int64_t)rows * (width / 8) + 255) / 256;
    TASC_REQUIRE(blocks < kMostBlocks, "kv4_append: %d rows of %d x %d channels are 2^35 and more", rows, c->n_kv_heads, c->head_dim);
    const dim3 grid((unsigned)blocks, 2);
    hipStream_t st = (hipStream_t)stream;
    with_hd(c->head_dim, [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        auto go = [&](auto kernel, auto* kk, auto* vv) { kernel<<<grid, dim3(256), 0, st>>>(a, kk, vv, k_stride, v_stride); };
        if (dtype == TASC_F32) go(vec ? &k_kv4_append<HD, float, true> : &k_kv4_append<HD, float, false>, (const float*)k, (const float*)v);
        else go(vec ? &k_kv4_append<HD, BF16, true> : &k_kv4_append<HD, BF16, false>, (const BF16*)k, (const BF16*)v);
    });
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

extern "C" tasc_status tasc_kv4_read(const tasc_kv4_cache* c, const int32_t* slots, int32_t rows, tasc_dtype dtype, void* k, void* v, void* stream) {
    tasc_status rc = check_cache("kv4_read", c);
    if (rc != TASC_OK) return rc;
    TASC_REQUIRE(rows >= 0, "kv4_read: %d rows", rows);
    if (rows == 0) return TASC_OK;
    TASC_REQUIRE(k && v && slots, "kv4_read: null argument");
    TASC_REQUIRE(dtype == TASC_F32 || dtype == TASC_BF16, "kv4_read: dtype %d", (int)dtype);
    TASC_REQUIRE((((uintptr_t)k | (uintptr_t)v) & 15) == 0, "kv4_read: outputs must be 16-byte aligned");
    const Kv4Rows a{(uint8_t*)c->pool, c->n_pages, c->n_kv_heads, rows, slots};
    const int64_t blocks = ((int64_t)rows * c->n_kv_heads * (c->head_dim / 8) + 255) / 256;
    TASC_REQUIRE(blocks < kMostBlocks, "kv4_read: %d rows of %d x %d channels are 2^35 and more", rows, c->n_kv_heads, c->head_dim);
    const dim3 grid((unsigned)blocks, 2);
    hipStream_t st = (hipStream_t)stream;
    with_hd(c->head_dim, [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        if (dtype == TASC_F32) k_kv4_read<HD, float><<<grid, dim3(256), 0, st>>>(a, (float*)k, (float*)v);
        else k_kv4_read<HD, BF16><<<grid, dim3(256), 0, st>>>(a, (BF16*)k, (BF16*)v);
    });
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

extern "C" size_t tasc_kv4_attention_workspace_bytes(int32_t batch, int32_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows,
                                                     int32_t max_kv) {
    if (batch < 1 || rows < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || !kv4_head_dim_ok(head_dim) || max_rows < 1 || max_kv < 0) return 0;
    const Kv4Order o = kv4_order(batch, n_kv_heads, (int64_t)max_rows * (n_heads / n_kv_heads), max_kv, kMostChunks, false);
    return o.chunks == 1 ? 0 : (size_t)o.chunks * rows * n_heads * (head_dim + 2) * sizeof(float);
}

extern "C" tasc_status tasc_kv4_attention(const tasc_kv4_cache* c, const tasc_kv4_attn* p, void* workspace, size_t ws_bytes, void* stream) {
    tasc_status rc = check_cache("kv4_attention", c);
    if (rc != TASC_OK) return rc;
    TASC_REQUIRE(p, "kv4_attention: null argument");
    TASC_REQUIRE(p->batch >= 0 && p->rows >= 0 && p->max_rows >= 0 && p->max_kv >= 0 && p->max_pages >= 1, "kv4_attention: batch %d, rows %d, max_rows %d, max_kv %d, max_pages %d",
                 p->batch, p->rows, p->max_rows, p->max_kv, p->max_pages);
    if (p->batch == 0 || p->rows == 0 || p->max_rows == 0) return TASC_OK;
    TASC_REQUIRE(p->q && p->out && p->table && p->row_off && p->kv_len, "kv4_attention: null argument");
    TASC_REQUIRE(p->n_heads >= 1 && p->n_heads % c->n_kv_heads == 0, "kv4_attention: %d query heads over %d KV heads", p->n_heads, c->n_kv_heads);
    TASC_REQUIRE((int64_t)p->batch * c->n_kv_heads <= 65535, "kv4_attention: batch %d x %d KV heads is beyond 65535", p->batch, c->n_kv_heads);
    TASC_REQUIRE(p->max_pages <= (1 << 26) && (int64_t)p->max_rows * p->n_heads < (int64_t)1 << 30, "kv4_attention: max_pages %d, max_rows %d", p->max_pages, p->max_rows);
    TASC_REQUIRE(((int64_t)p->max_rows * (p->n_heads / c->n_kv_heads) + 127) / 128 * p->batch * c->n_kv_heads < kMostBlocks,
                 "kv4_attention: batch %d of up to %d rows of %d heads is beyond 2^31", p->batch, p->max_rows, p->n_heads);
    const int64_t width = (int64_t)p->n_heads * c->head_dim;
    TASC_REQUIRE(p->q_stride >= 0 && p->out_stride >= width, "kv4_attention: row strides %lld, %lld of rows of %lld", (long long)p->q_stride, (long long)p->out_stride,
                 (long long)width);
    TASC_REQUIRE(((uintptr_t)p->q & 15) == 0 && ((uintptr_t)p->out & 15) == 0 && p->q_stride % 8 == 0 && p->out_stride % 8 == 0,
                 "kv4_attention: rows of queries and results must be 16-byte aligned");
    const Kv4Order order = kv4_order(p->batch, c->n_kv_heads, (int64_t)p->max_rows * (p->n_heads / c->n_kv_heads), p->max_kv, kMostChunks, false);
    const size_t n = (size_t)order.chunks * p->rows * p->n_heads, need = order.chunks == 1 ? 0 : n * (c->head_dim + 2) * sizeof(float);
    if (need > 0 && (!workspace || ws_bytes < need)) {
        tasc_set_error("kv4_attention: workspace of %zu of %zu bytes", workspace ? ws_bytes : 0, need);
        return TASC_ENOMEM;
    }
    TASC_REQUIRE(need == 0 || ((uintptr_t)workspace & 15) == 0, "kv4_attention: the workspace must be 16-byte aligned");
    Kv4Attn a{};
    a.pool = (const uint8_t*)c->pool;
    a.n_pages = c->n_pages; a.max_pages = p->max_pages; a.Hkv = c->n_kv_heads; a.H = p->n_heads; a.batch = p->batch; a.rows = p->rows;
    a.max_rows = p->max_rows;
    a.q = (const BF16*)p->q; a.out = (BF16*)p->out; a.q_stride = p->q_stride; a.out_stride = p->out_stride;
    a.table = p->table; a.row_off = p->row_off; a.kv_len = p->kv_len;
    a.scale = p->scale;
    a.part_o = (float*)workspace;
    a.part_ml = order.chunks == 1 ? nullptr : (float*)workspace + n * c->head_dim;
    return tasc_kv4_attend(a, c->head_dim, order, (hipStream_t)stream);
}
