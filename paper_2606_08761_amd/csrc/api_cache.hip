// C ABI front end of the paged key-value cache and its attention: argument
// validation (before any HIP call), device check and dispatch.  See
// include/apex4.h for the contract.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4.h"
#include "apex4_internal.h"
#include "kv_cache.h"

namespace {

using apex4::AttnArgs;
using apex4::KvView;
using apex4::PageTable;
using apex4::Rotary;

constexpr int64_t kMaxPages = 1ll << 30, kMaxWidth = 1ll << 20, kMaxLen = 1ll << 30, kMaxCount = 1ll << 24, kMaxRows = 1ll << 27;
constexpr int64_t kMaxPageBytes = 1ll << 30;  // offsets inside a page are 32 bits

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool present(const void* p, int64_t n) { return p != nullptr || n == 0; }
int64_t min64(int64_t a, int64_t b) { return a < b ? a : b; }

int shift_of(int64_t page) {
    for (int s = 4; s <= 10; ++s)
        if (page == (1ll << s)) return s;
    return -1;
}

int check_geometry(int cache, int64_t kv_heads, int64_t D, int64_t page) {
    if (cache != APEX4_KV_FP16 && cache != APEX4_KV_INT4) return APEX4_ERR_SHAPE;
    if (kv_heads < 1 || kv_heads > 65536 || (D != 64 && D != 128) || shift_of(page) < 0) return APEX4_ERR_SHAPE;
    return apex4::kv_page_bytes(cache == APEX4_KV_INT4, kv_heads, D, page) <= kMaxPageBytes ? APEX4_OK : APEX4_ERR_SHAPE;
}

// The cache's arguments; pointers and alignment are checked by the callers in
// the order that the header states.
int make_view(KvView& c, const void* k_pages, const void* v_pages, int64_t n_pages, const int32_t* table, int64_t width,
              const int32_t* kv_len, int64_t B, int64_t max_len, int64_t kv_heads, int64_t D, int64_t page, int cache) {
    const int rc = check_geometry(cache, kv_heads, D, page);
    if (rc) return rc;
    if (n_pages < 1 || n_pages > kMaxPages || width < 1 || width > kMaxWidth || B < 0 || B > kMaxCount) return APEX4_ERR_SHAPE;
    if (max_len < 0 || max_len > kMaxLen) return APEX4_ERR_SHAPE;
    c.k = static_cast<const uint8_t*>(k_pages);
    c.v = static_cast<const uint8_t*>(v_pages);
    c.table = table;
    c.kv_len = kv_len;
    c.n_pages = n_pages;
    c.i4 = cache == APEX4_KV_INT4;
    c.page_bytes = apex4::kv_page_bytes(c.i4, kv_heads, D, page);
    c.max_len = max_len;
    c.width = static_cast<int>(width);
    c.page_shift = shift_of(page);
    c.B = static_cast<int>(B);
    c.kv_heads = static_cast<int>(kv_heads);
    c.D = static_cast<int>(D);
    return APEX4_OK;
}

int check_view_pointers(const KvView& c) {
    if (!aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.table, 4) || !aligned(c.kv_len, 4)) return APEX4_ERR_ALIGN;
    return APEX4_OK;
}

// A row of `heads` heads every `stride` elements.
int check_rows(int64_t T, int64_t heads, int64_t D, int64_t stride) {
    if (T < 0 || T > kMaxCount || T * heads > kMaxRows) return APEX4_ERR_SHAPE;  // heads <= 65536: no wrap
    if (stride < heads * D || stride % 8 != 0 || stride > (1ll << 40)) return APEX4_ERR_SHAPE;
    return APEX4_OK;
}

// Whether T rows of n elements of x and of out_n of out share memory.  Of unequal strides the
// whole ranges count.
bool overlap(const void* x, int64_t x_stride, int64_t n, const void* out, int64_t out_stride, int64_t out_n, int64_t T) {
    if (T < 1) return false;
    const int64_t a = static_cast<int64_t>(reinterpret_cast<uintptr_t>(x) / 2), b = static_cast<int64_t>(reinterpret_cast<uintptr_t>(out) / 2);
    if (a + (T - 1) * x_stride + n <= b || b + (T - 1) * out_stride + out_n <= a) return false;
    if (T == 1 || x_stride != out_stride) return true;
    const int64_t d = ((b - a) % x_stride + x_stride) % x_stride;  // from a row of x on to the next one of out
    return d < n || d + out_n > x_stride;
}

int make_rotary(Rotary& r, const double* freq, int64_t D, int64_t rot, int layout, double mag) {
    if (rot < 2 || rot > D || rot % 2 != 0) return APEX4_ERR_SHAPE;
    if (layout != APEX4_ROPE_HALF && layout != APEX4_ROPE_INTERLEAVED) return APEX4_ERR_SHAPE;
    if (!(mag > 0.0) || mag > 3.4e38) return APEX4_ERR_SHAPE;
    r.freq = freq;
    r.mag = mag;
    r.rot = static_cast<int>(rot);
    r.interleaved = layout == APEX4_ROPE_INTERLEAVED;
    return APEX4_OK;
}

int make_attn(AttnArgs& a, const KvView& c, const void* q, int64_t q_stride, const int32_t* q_start, int64_t T,
              int64_t max_q, int64_t heads, int64_t window, int64_t sinks, float scale, void* out) {
    if (heads < 1 || heads > 65536 || heads % c.kv_heads != 0) return APEX4_ERR_SHAPE;
    if (max_q < 0 || max_q > kMaxCount) return APEX4_ERR_SHAPE;
    const int rc = check_rows(T, heads, c.D, q_stride);
    if (rc) return rc;
    if (window < 0 || sinks < 0 || !(scale > 0.f) || scale > 3.4e38f) return APEX4_ERR_SHAPE;
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.q_start = q_start;
    a.T = T;
    a.max_q = min64(max_q, T);  // a sequence has no more
    a.heads = static_cast<int>(heads);
    a.group = static_cast<int>(heads / c.kv_heads);
    a.window = static_cast<int>(min64(window, kMaxLen));
    a.sinks = static_cast<int>(min64(sinks, kMaxLen));
    a.scale = scale;
    a.out = static_cast<uint16_t*>(out);
    return APEX4_OK;
}

// The workspace that serves either kind of cache.
int largest(KvView c, const AttnArgs& a, bool empty, int64_t (*size)(const KvView&, const AttnArgs&), int64_t* bytes) {
    int64_t most = 0;
    for (const bool i4 : {false, true}) {
        if (empty) break;
        c.i4 = i4;
        const int64_t need = size(c, a);
        if (need < 0) return APEX4_ERR_SHAPE;
        most = need > most ? need : most;
    }
    *bytes = most;
    return APEX4_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? APEX4_OK : APEX4_ERR_LAUNCH; }

int make_table(PageTable& p, int32_t* table, int64_t slots, int64_t width, int32_t* kv_len, int32_t* refs, int64_t n_pages,
               int64_t n, int64_t page) {
    if (slots < 1 || slots > kMaxCount || width < 1 || width > kMaxWidth || n_pages < 1 || n_pages > kMaxPages) return APEX4_ERR_SHAPE;
    if (n < 0 || n > kMaxCount || shift_of(page) < 0) return APEX4_ERR_SHAPE;
    p.table = table;
    p.kv_len = kv_len;
    p.refs = refs;
    p.slots = static_cast<int>(slots);
    p.width = static_cast<int>(width);
    p.n_pages = static_cast<int>(n_pages);
    p.page_shift = shift_of(page);
    return APEX4_OK;
}

int check_pool(const void* pool, int64_t planes, int64_t page_bytes) {
    if (planes < 1 || planes > 65536 || page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > kMaxPageBytes) return APEX4_ERR_SHAPE;
    return aligned(pool, 16) ? APEX4_OK : APEX4_ERR_ALIGN;
}

}  // namespace

using apex4::check_device;

extern "C" {

int apex4_kv_page_bytes(int cache, int64_t kv_heads, int64_t head_dim, int64_t page, int64_t* bytes) {
    if (!bytes) return APEX4_ERR_NULL;
    const int rc = check_geometry(cache, kv_heads, head_dim, page);
    if (rc) return rc;
    *bytes = apex4::kv_page_bytes(cache == APEX4_KV_INT4, kv_heads, head_dim, page);
    return APEX4_OK;
}

int apex4_kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* q_start, int64_t T,
                    void* k_pages, void* v_pages, int64_t n_pages, const int32_t* table, int64_t width,
                    const int32_t* kv_len, int64_t B, int64_t kv_heads, int64_t head_dim, int64_t page, int cache,
                    void* stream) {
    if (!present(k, T) || !present(v, T) || !k_pages || !v_pages || !present(table, B) || !present(kv_len, B)) return APEX4_ERR_NULL;
    KvView c;
    int rc = make_view(c, k_pages, v_pages, n_pages, table, width, kv_len, B, kMaxLen, kv_heads, head_dim, page, cache);
    if (rc) return rc;
    if ((rc = check_rows(T, kv_heads, head_dim, k_stride)) || (rc = check_rows(T, kv_heads, head_dim, v_stride))) return rc;
    if (T > 0 && (q_start ? B < 1 : T != B)) return APEX4_ERR_SHAPE;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(q_start, 4)) return APEX4_ERR_ALIGN;
    if ((rc = check_view_pointers(c)) || (rc = check_device())) return rc;
    if (T == 0) return APEX4_OK;
    return status_of(apex4::launch_kv_append(c, static_cast<const uint16_t*>(k), k_stride, static_cast<const uint16_t*>(v),
                                             v_stride, q_start, T, static_cast<hipStream_t>(stream)));
}

int apex4_rope(const void* x, int64_t x_stride, const int32_t* positions, int64_t T, int64_t heads, int64_t head_dim,
               const double* freq, int64_t rot, int layout, double mag, void* out, int64_t out_stride, void* stream) {
    if (!present(x, T) || !present(positions, T) || !freq || !present(out, T)) return APEX4_ERR_NULL;
    Rotary r;
    if (heads < 1 || heads > 65536 || head_dim < 8 || head_dim > 512 || head_dim % 8 != 0) return APEX4_ERR_SHAPE;
    int rc = make_rotary(r, freq, head_dim, rot, layout, mag);
    if (rc) return rc;
    if ((rc = check_rows(T, heads, head_dim, x_stride)) || (rc = check_rows(T, heads, head_dim, out_stride))) return rc;
    if (T > 1 && x == out && x_stride != out_stride) return APEX4_ERR_SHAPE;
    if (!aligned(x, 16) || !aligned(positions, 4) || !aligned(freq, 8) || !aligned(out, 16)) return APEX4_ERR_ALIGN;
    if (x != out && overlap(x, x_stride, heads * head_dim, out, out_stride, heads * head_dim, T)) return APEX4_ERR_SHAPE;
    if ((rc = check_device())) return rc;
    if (T == 0) return APEX4_OK;
    return status_of(apex4::launch_rope(static_cast<const uint16_t*>(x), x_stride, positions, T, static_cast<int>(heads),
                                        static_cast<int>(head_dim), r, static_cast<uint16_t*>(out), out_stride,
                                        static_cast<hipStream_t>(stream)));
}

int apex4_kv_append_rope(const void* q, int64_t q_stride, int64_t heads, void* q_out, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, const int32_t* q_start, int64_t T, const int32_t* positions,
                         const double* freq, int64_t rot, int layout, double mag, void* k_pages, void* v_pages,
                         int64_t n_pages, const int32_t* table, int64_t width, const int32_t* kv_len, int64_t B,
                         int64_t kv_heads, int64_t head_dim, int64_t page, int cache, void* stream) {
    const int64_t queries = heads == 0 ? 0 : T;
    if (!present(q, queries) || !present(q_out, queries) || !present(k, T) || !present(v, T) || !freq || !k_pages || !v_pages ||
        !present(table, B) || !present(kv_len, B))
        return APEX4_ERR_NULL;
    KvView c;
    Rotary r;
    int rc = make_view(c, k_pages, v_pages, n_pages, table, width, kv_len, B, kMaxLen, kv_heads, head_dim, page, cache);
    if (rc || (rc = make_rotary(r, freq, head_dim, rot, layout, mag))) return rc;
    if (heads < 0 || heads > 65536) return APEX4_ERR_SHAPE;
    if (heads && (rc = check_rows(T, heads, head_dim, q_stride))) return rc;
    if ((rc = check_rows(T, kv_heads, head_dim, k_stride)) || (rc = check_rows(T, kv_heads, head_dim, v_stride))) return rc;
    if (T > 0 && (q_start ? B < 1 : T != B)) return APEX4_ERR_SHAPE;
    if (heads && q == q_out && T > 0) return APEX4_ERR_SHAPE;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(q_start, 4) || !aligned(positions, 4) || !aligned(freq, 8)) return APEX4_ERR_ALIGN;
    if (heads && (!aligned(q, 16) || !aligned(q_out, 16))) return APEX4_ERR_ALIGN;
    if ((rc = check_view_pointers(c))) return rc;
    const int64_t row = heads * head_dim, kv_row = kv_heads * head_dim;
    if (heads && (overlap(q, q_stride, row, q_out, row, row, T) || overlap(k, k_stride, kv_row, q_out, row, row, T) ||
                  overlap(v, v_stride, kv_row, q_out, row, row, T)))
        return APEX4_ERR_SHAPE;
    if ((rc = check_device())) return rc;
    if (T == 0) return APEX4_OK;
    apex4::RopeRows a;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.heads = static_cast<int>(heads);
    a.positions = positions;
    return status_of(apex4::launch_kv_append_rope(c, a, q_start, T, r, static_cast<hipStream_t>(stream)));
}

int apex4_kv_gather(const void* k_pages, const void* v_pages, int64_t n_pages, const int32_t* table, int64_t width,
                    const int32_t* kv_len, int64_t B, int64_t kv_heads, int64_t head_dim, int64_t page, int cache,
                    const int32_t* q_start, int64_t T, void* k, void* v, void* stream) {
    if (!present(k, T) || !present(v, T) || !k_pages || !v_pages || !present(table, B) || !present(kv_len, B)) return APEX4_ERR_NULL;
    KvView c;
    int rc = make_view(c, k_pages, v_pages, n_pages, table, width, kv_len, B, kMaxLen, kv_heads, head_dim, page, cache);
    if (rc) return rc;
    if ((rc = check_rows(T, kv_heads, head_dim, kv_heads * head_dim))) return rc;
    if (T > 0 && (q_start ? B < 1 : T != B)) return APEX4_ERR_SHAPE;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(q_start, 4)) return APEX4_ERR_ALIGN;
    if ((rc = check_view_pointers(c)) || (rc = check_device())) return rc;
    if (T == 0) return APEX4_OK;
    return status_of(apex4::launch_kv_gather(c, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), q_start, T,
                                             static_cast<hipStream_t>(stream)));
}

int apex4_attn_decode_workspace_size(int64_t B, int64_t width, int64_t max_len, int64_t heads, int64_t kv_heads,
                                     int64_t head_dim, int64_t page, int64_t window, int64_t sinks, int64_t* bytes) {
    if (!bytes) return APEX4_ERR_NULL;
    KvView c;
    AttnArgs a;
    int rc = make_view(c, nullptr, nullptr, 1, nullptr, width, nullptr, B, max_len, kv_heads, head_dim, page, APEX4_KV_FP16);
    if (rc) return rc;
    if ((rc = make_attn(a, c, nullptr, heads * head_dim, nullptr, B, 1, heads, window, sinks, 1.f, nullptr))) return rc;
    if ((rc = check_device())) return rc;
    return largest(c, a, B == 0, apex4::attn_decode_workspace, bytes);
}

int apex4_attn_decode(const void* q, int64_t q_stride, const void* k_pages, const void* v_pages, int64_t n_pages,
                      const int32_t* table, int64_t width, const int32_t* kv_len, int64_t B, int64_t max_len,
                      int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t page, int cache, int64_t window,
                      int64_t sinks, float scale, void* out, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!present(q, B) || !k_pages || !v_pages || !present(table, B) || !present(kv_len, B) || !present(out, B)) return APEX4_ERR_NULL;
    KvView c;
    AttnArgs a;
    int rc = make_view(c, k_pages, v_pages, n_pages, table, width, kv_len, B, max_len, kv_heads, head_dim, page, cache);
    if (rc) return rc;
    if ((rc = make_attn(a, c, q, q_stride, nullptr, B, 1, heads, window, sinks, scale, out))) return rc;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16)) return APEX4_ERR_ALIGN;
    if ((rc = check_view_pointers(c)) || (rc = check_device())) return rc;
    if (B == 0) return APEX4_OK;
    const int64_t need = apex4::attn_decode_workspace(c, a);
    if (need < 0) return APEX4_ERR_SHAPE;
    if (need > 0 && (!workspace || workspace_bytes < need)) return APEX4_ERR_WORKSPACE;
    a.workspace = workspace;
    return status_of(apex4::launch_attn_decode(c, a, static_cast<hipStream_t>(stream)));
}

int apex4_attn_prefill_workspace_size(int64_t T, int64_t B, int64_t max_q, int64_t width, int64_t max_len, int64_t heads,
                                      int64_t kv_heads, int64_t head_dim, int64_t page, int64_t window, int64_t sinks,
                                      int64_t* bytes) {
    if (!bytes) return APEX4_ERR_NULL;
    KvView c;
    AttnArgs a;
    int rc = make_view(c, nullptr, nullptr, 1, nullptr, width, nullptr, B, max_len, kv_heads, head_dim, page, APEX4_KV_FP16);
    if (rc) return rc;
    if ((rc = make_attn(a, c, nullptr, heads * head_dim, nullptr, T, max_q, heads, window, sinks, 1.f, nullptr))) return rc;
    if ((rc = check_device())) return rc;
    return largest(c, a, T == 0 || B == 0 || max_q == 0, apex4::attn_prefill_workspace, bytes);
}

int apex4_attn_prefill(const void* q, int64_t q_stride, const int32_t* q_start, int64_t T, int64_t max_q,
                       const void* k_pages, const void* v_pages, int64_t n_pages, const int32_t* table, int64_t width,
                       const int32_t* kv_len, int64_t B, int64_t max_len, int64_t heads, int64_t kv_heads,
                       int64_t head_dim, int64_t page, int cache, int64_t window, int64_t sinks, float scale, void* out,
                       void* workspace, int64_t workspace_bytes, void* stream) {
    if (!present(q, T) || !present(q_start, T) || !k_pages || !v_pages || !present(table, B) || !present(kv_len, B) || !present(out, T))
        return APEX4_ERR_NULL;
    KvView c;
    AttnArgs a;
    int rc = make_view(c, k_pages, v_pages, n_pages, table, width, kv_len, B, max_len, kv_heads, head_dim, page, cache);
    if (rc) return rc;
    if ((rc = make_attn(a, c, q, q_stride, q_start, T, max_q, heads, window, sinks, scale, out))) return rc;
    if (T > 0 && (B < 1 || max_q < 1)) return APEX4_ERR_SHAPE;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(q_start, 4)) return APEX4_ERR_ALIGN;
    if ((rc = check_view_pointers(c)) || (rc = check_device())) return rc;
    if (T == 0) return APEX4_OK;
    const int64_t need = apex4::attn_prefill_workspace(c, a);
    if (need < 0) return APEX4_ERR_SHAPE;
    if (need > 0 && (!workspace || workspace_bytes < need)) return APEX4_ERR_WORKSPACE;
    a.workspace = workspace;
    return status_of(apex4::launch_attn_prefill(c, a, static_cast<hipStream_t>(stream)));
}

int apex4_pages_workspace_size(int64_t n_pages, int64_t n, int64_t* bytes) {
    if (!bytes) return APEX4_ERR_NULL;
    if (n_pages < 1 || n_pages > kMaxPages || n < 0 || n > kMaxCount) return APEX4_ERR_SHAPE;
    *bytes = apex4::pages_work_words(n_pages, n) * 4;
    return APEX4_OK;
}

int apex4_pages_reserve(int32_t* table, int64_t slots, int64_t width, int32_t* kv_len, int32_t* refs, int64_t n_pages,
                        const int32_t* seqs, const int32_t* new_len, int64_t n, int64_t page, int32_t* status,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    if (!table || !kv_len || !refs || !present(seqs, n) || !present(new_len, n) || !status) return APEX4_ERR_NULL;
    PageTable p;
    int rc = make_table(p, table, slots, width, kv_len, refs, n_pages, n, page);
    if (rc) return rc;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(refs, 4) || !aligned(seqs, 4) || !aligned(new_len, 4) ||
        !aligned(status, 4) || !aligned(workspace, 16))
        return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (!workspace || workspace_bytes < apex4::pages_work_words(n_pages, n) * 4) return APEX4_ERR_WORKSPACE;
    return status_of(apex4::launch_pages_reserve(p, seqs, new_len, static_cast<int>(n), status,
                                                 static_cast<int32_t*>(workspace), static_cast<hipStream_t>(stream)));
}

int apex4_pages_fork(void* pool, int64_t planes, int64_t page_bytes, int32_t* table, int64_t slots, int64_t width,
                     int32_t* kv_len, int32_t* refs, int64_t n_pages, const int32_t* parents, const int32_t* children,
                     int64_t n, int64_t page, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!pool || !table || !kv_len || !refs || !present(parents, n) || !present(children, n) || !status) return APEX4_ERR_NULL;
    PageTable p;
    int rc = make_table(p, table, slots, width, kv_len, refs, n_pages, n, page);
    if (rc || (rc = check_pool(pool, planes, page_bytes))) return rc;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(refs, 4) || !aligned(parents, 4) || !aligned(children, 4) ||
        !aligned(status, 4) || !aligned(workspace, 16))
        return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (!workspace || workspace_bytes < apex4::pages_work_words(n_pages, n) * 4) return APEX4_ERR_WORKSPACE;
    return status_of(apex4::launch_pages_fork(p, static_cast<uint8_t*>(pool), static_cast<int>(planes), page_bytes, parents,
                                              children, static_cast<int>(n), status, static_cast<int32_t*>(workspace),
                                              static_cast<hipStream_t>(stream)));
}

int apex4_pages_free(int32_t* table, int64_t slots, int64_t width, int32_t* kv_len, int32_t* refs, int64_t n_pages,
                     const int32_t* seqs, int64_t n, void* stream) {
    if (!table || !kv_len || !refs || !present(seqs, n)) return APEX4_ERR_NULL;
    PageTable p;
    int rc = make_table(p, table, slots, width, kv_len, refs, n_pages, n, 16);
    if (rc) return rc;
    if (!aligned(table, 4) || !aligned(kv_len, 4) || !aligned(refs, 4) || !aligned(seqs, 4)) return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (n == 0) return APEX4_OK;
    return status_of(apex4::launch_pages_free(p, seqs, static_cast<int>(n), static_cast<hipStream_t>(stream)));
}

int apex4_pages_compact(void* pool, int64_t planes, int64_t page_bytes, int32_t* table, int64_t slots, int64_t width,
                        int32_t* refs, int64_t n_pages, int32_t* status, void* workspace, int64_t workspace_bytes,
                        void* stream) {
    if (!pool || !table || !refs || !status) return APEX4_ERR_NULL;
    PageTable p;
    int rc = make_table(p, table, slots, width, nullptr, refs, n_pages, 0, 16);
    if (rc || (rc = check_pool(pool, planes, page_bytes))) return rc;
    if (!aligned(table, 4) || !aligned(refs, 4) || !aligned(status, 4) || !aligned(workspace, 16)) return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (!workspace || workspace_bytes < apex4::pages_work_words(n_pages, 0) * 4) return APEX4_ERR_WORKSPACE;
    return status_of(apex4::launch_pages_compact(p, static_cast<uint8_t*>(pool), static_cast<int>(planes), page_bytes, status,
                                                 static_cast<int32_t*>(workspace), static_cast<hipStream_t>(stream)));
}

int apex4_pages_copy(void* pool, int64_t planes, int64_t page_bytes, int64_t n_pages, const int32_t* src, const int32_t* dst,
                     int64_t n, void* stream) {
    if (!pool || !present(src, n) || !present(dst, n)) return APEX4_ERR_NULL;
    if (n_pages < 1 || n_pages > kMaxPages || n < 0 || n > kMaxCount) return APEX4_ERR_SHAPE;
    int rc = check_pool(pool, planes, page_bytes);
    if (rc) return rc;
    if (!aligned(src, 4) || !aligned(dst, 4)) return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (n == 0) return APEX4_OK;
    return status_of(apex4::launch_pages_copy(static_cast<uint8_t*>(pool), static_cast<int>(planes), page_bytes,
                                              static_cast<int>(n_pages), src, dst, static_cast<int>(n),
                                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
