// C-ABI entry points of the operators between the projections (include/qblora.h): host-side validation and descriptions.
#include <cmath>

#include "decoder.h"

using namespace qblora;

namespace {

// log2 of a page size the cache knows; -1 otherwise
int page_shift_of(int page) {
    for (int s = 4; s <= 8; ++s)
        if (page == 1 << s) return s;
    return -1;
}
bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int64_t kMostPositions = (int64_t)1 << 30;       // positions of a request and tokens of a call: 32-bit arithmetic

constexpr int32_t kMostRequests = 1 << 30;                 // they are counted in steps of up to 2^19, in 32 bits

int check_cache(const qblora_kv_cache* c) {
    if (!c || !c->k || !c->v) return QBLORA_ERR_NULL;
    if (c->pages <= 0 || c->heads <= 0 || c->head_dim <= 0 || c->page <= 0) return QBLORA_ERR_SHAPE;
    if (page_shift_of(c->page) < 0) return QBLORA_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return QBLORA_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return QBLORA_ERR_SHAPE;
    return QBLORA_OK;
}

int check_rope(const qblora_rope* r, int32_t heads, int32_t kv_heads, int32_t head_dim, bool keys, int64_t T) {
    if (!r || !r->freq) return QBLORA_ERR_NULL;
    if (T < 0 || heads <= 0 || (keys && kv_heads <= 0) || head_dim <= 0) return QBLORA_ERR_SHAPE;
    if (r->rot <= 0 || r->rot % 2 != 0 || r->rot > head_dim) return QBLORA_ERR_SHAPE;
    if (head_dim > 1024 || (int64_t)(heads + (int64_t)kv_heads) * head_dim > INT32_MAX / 8 || T > kMostPositions)
        return QBLORA_ERR_UNSUPPORTED;
    return QBLORA_OK;
}

int rope_both(const qblora_rope* rope, float sign, const qblora_bf16* q, int64_t ldq, int32_t heads, const qblora_bf16* k,
              int64_t ldk, int32_t kv_heads, int32_t head_dim, const int32_t* positions, int64_t T, qblora_bf16* q_out,
              int64_t ldq_out, qblora_bf16* k_out, int64_t ldk_out, void* stream) {
    const int rc = check_rope(rope, heads, kv_heads, head_dim, k != nullptr, T);
    if (rc) return rc;
    if (!q || !q_out || !positions || (k && !k_out)) return T ? QBLORA_ERR_NULL : QBLORA_OK;
    const int64_t wq = (int64_t)heads * head_dim, wk = (int64_t)kv_heads * head_dim;
    if (ldq < wq || ldq_out < wq || (k && (ldk < wk || ldk_out < wk))) return QBLORA_ERR_SHAPE;
    if (T == 0) return QBLORA_OK;
    RopeDesc d{};
    d.freq = rope->freq; d.rot = rope->rot; d.interleaved = rope->interleaved != 0; d.scale = rope->scale; d.sign = sign;
    d.q = q; d.ldq = ldq; d.heads = heads; d.k = k; d.ldk = ldk; d.kv_heads = k ? kv_heads : 0; d.head_dim = head_dim;
    d.positions = positions; d.T = T; d.q_out = q_out; d.ldq_out = ldq_out; d.k_out = k_out; d.ldk_out = ldk_out;
    return launch_rope(d, as_stream(stream));
}

int check_norm(const void* total, const void* w, int64_t T, int32_t d) {
    if (T < 0 || d <= 0) return QBLORA_ERR_SHAPE;
    if (d > 16384 || T > INT32_MAX) return QBLORA_ERR_UNSUPPORTED;
    if (!w || (T && !total)) return QBLORA_ERR_NULL;
    return QBLORA_OK;
}

}  // namespace

extern "C" {

int qblora_page_tables(const int32_t* context, const int32_t* fresh, int32_t n, int32_t page, const int32_t* free_pages,
                       int32_t n_free, int32_t* table, int32_t width, int64_t tokens, int32_t* starts, int32_t* positions,
                       int64_t* slots, int32_t* taken, void* stream) {
    if (n < 0 || n_free < 0 || width < 0 || tokens < 0 || tokens > INT32_MAX || page <= 0) return QBLORA_ERR_SHAPE;
    if ((int64_t)n * width > INT32_MAX) return QBLORA_ERR_SHAPE;
    if (page_shift_of(page) < 0 || n > kMostRequests) return QBLORA_ERR_UNSUPPORTED;
    if (!starts || !taken || (n && (!context || !fresh)) || (n && width && !table) || (n_free && !free_pages) ||
        (tokens && (!positions || !slots)))
        return QBLORA_ERR_NULL;
    TablesDesc d{};
    d.context = context; d.fresh = fresh; d.n = n; d.page_shift = page_shift_of(page);
    d.free_pages = free_pages; d.n_free = n_free; d.table = table; d.width = width; d.tokens = (int)tokens;
    d.starts = starts; d.positions = positions; d.slots = slots; d.taken = taken;
    return launch_page_tables(d, as_stream(stream));
}

int qblora_rope_fwd(const qblora_rope* rope, const qblora_bf16* q, int64_t ldq, int32_t heads, const qblora_bf16* k,
                    int64_t ldk, int32_t kv_heads, int32_t head_dim, const int32_t* positions, int64_t T,
                    qblora_bf16* q_out, int64_t ldq_out, qblora_bf16* k_out, int64_t ldk_out, void* stream) {
    return rope_both(rope, 1.0f, q, ldq, heads, k, ldk, kv_heads, head_dim, positions, T, q_out, ldq_out, k_out, ldk_out, stream);
}

int qblora_rope_bwd(const qblora_rope* rope, const qblora_bf16* dq, int64_t lddq, int32_t heads, const qblora_bf16* dk,
                    int64_t lddk, int32_t kv_heads, int32_t head_dim, const int32_t* positions, int64_t T,
                    qblora_bf16* dq_out, int64_t lddq_out, qblora_bf16* dk_out, int64_t lddk_out, void* stream) {
    return rope_both(rope, -1.0f, dq, lddq, heads, dk, lddk, kv_heads, head_dim, positions, T, dq_out, lddq_out, dk_out,
                     lddk_out, stream);
}

int qblora_rope_cache(const qblora_rope* rope, const qblora_bf16* q, int64_t ldq, int32_t heads, const qblora_bf16* k,
                      int64_t ldk, const qblora_bf16* v, int64_t ldv, const int32_t* positions, const int64_t* slots,
                      int64_t T, qblora_bf16* q_out, int64_t ldq_out, const qblora_kv_cache* cache, void* stream) {
    int rc = check_cache(cache);
    if (rc) return rc;
    rc = check_rope(rope, heads, cache->heads, cache->head_dim, true, T);
    if (rc) return rc;
    if (!q || !k || !v || !positions || !slots || !q_out) return T ? QBLORA_ERR_NULL : QBLORA_OK;
    const int64_t wq = (int64_t)heads * cache->head_dim, wk = (int64_t)cache->heads * cache->head_dim;
    if (ldq < wq || ldq_out < wq || ldk < wk || ldv < wk) return QBLORA_ERR_SHAPE;
    if (T == 0) return QBLORA_OK;
    RopeDesc d{};
    d.freq = rope->freq; d.rot = rope->rot; d.interleaved = rope->interleaved != 0; d.scale = rope->scale; d.sign = 1.0f;
    d.q = q; d.ldq = ldq; d.heads = heads; d.k = k; d.ldk = ldk; d.kv_heads = cache->heads; d.head_dim = cache->head_dim;
    d.positions = positions; d.T = T; d.q_out = q_out; d.ldq_out = ldq_out;
    d.v = v; d.ldv = ldv; d.slots = slots; d.kc = cache->k; d.vc = cache->v;
    d.cache_slots = (int64_t)cache->pages * cache->page; d.page_shift = page_shift_of(cache->page);
    return launch_rope(d, as_stream(stream));
}

int qblora_rope_frequencies(int32_t rot, double base, int32_t kind, double factor, double original, double low, double high,
                            float* freq, float* scale) {
    if (!freq) return QBLORA_ERR_NULL;
    if (rot <= 0 || rot % 2 != 0 || !(base > 0.0)) return QBLORA_ERR_SHAPE;
    if (kind < QBLORA_ROPE_PLAIN || kind > QBLORA_ROPE_BY_PARTS) return QBLORA_ERR_UNSUPPORTED;
    if (kind != QBLORA_ROPE_PLAIN && !(factor > 0.0)) return QBLORA_ERR_SHAPE;
    if (kind == QBLORA_ROPE_BASE && rot < 4) return QBLORA_ERR_SHAPE;
    if (kind == QBLORA_ROPE_BY_PARTS && !(original > 0.0 && low < high)) return QBLORA_ERR_SHAPE;
    if (kind == QBLORA_ROPE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int j = 0; j < rot / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rot);
        if (kind == QBLORA_ROPE_LINEAR) f /= factor;
        if (kind == QBLORA_ROPE_BY_PARTS) {
            const double turns = original * f / 6.283185307179586477;
            const double g = std::fmin(std::fmax((turns - low) / (high - low), 0.0), 1.0);
            f *= g + (1.0 - g) / factor;
        }
        freq[j] = (float)f;
    }
    if (scale) *scale = kind == QBLORA_ROPE_BY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return QBLORA_OK;
}

size_t qblora_paged_attention_workspace_bytes(const qblora_kv_cache* cache, int32_t heads, int32_t max_new) {
    if (!cache || cache->heads <= 0 || heads <= 0 || heads % cache->heads != 0 || cache->head_dim <= 0) return 0;
    return attention_part_bytes(cache->head_dim, cache->heads, heads / cache->heads, max_new);
}

int qblora_paged_attention(const qblora_bf16* q, int64_t ldq, int32_t heads, const qblora_kv_cache* cache,
                           const int32_t* table, int32_t width, const int32_t* starts, const int32_t* context, int32_t n,
                           int64_t T, float scale, int32_t window, int32_t max_new, qblora_bf16* out, int64_t ldo, float* lse,
                           void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_cache(cache);
    if (rc) return rc;
    if (n < 0 || T < 0 || width < 0 || window < 0 || max_new < 0 || heads <= 0 || heads % cache->heads != 0)
        return QBLORA_ERR_SHAPE;
    if (n > kMostRequests || T > kMostPositions || (int64_t)width * cache->page > kMostPositions || window > kMostPositions ||
        T * (heads / cache->heads) > INT32_MAX || cache->heads > 65535 ||
        heads / cache->heads > 32768)
        return QBLORA_ERR_UNSUPPORTED;
    if (T == 0 || n == 0) return QBLORA_OK;
    if (!q || !out || !starts || !context || (width && !table)) return QBLORA_ERR_NULL;
    const int64_t row = (int64_t)heads * cache->head_dim;
    if (ldq < row || ldo < row || ldq % 8 != 0 || ldo % 8 != 0 || !aligned(q, 16) || !aligned(out, 16)) return QBLORA_ERR_SHAPE;
    if (!workspace || workspace_bytes < qblora_paged_attention_workspace_bytes(cache, heads, max_new)) return QBLORA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QBLORA_ERR_SHAPE;
    AttnDesc d{};
    d.q = q; d.ldq = ldq; d.heads = heads; d.kv_heads = cache->heads; d.group = heads / cache->heads;
    d.group_magic = (uint32_t)(((uint64_t)1 << 32) / (uint32_t)d.group + 1);
    d.kc = cache->k; d.vc = cache->v; d.pages = cache->pages; d.page_shift = page_shift_of(cache->page);
    d.head_dim = cache->head_dim; d.table = table; d.width = width; d.starts = starts; d.context = context;
    d.n = n; d.T = (int)T; d.scale_log2 = scale * 1.44269504088896340736f; d.window = window; d.max_new = max_new;
    d.out = out; d.ldo = ldo; d.lse = lse; d.part = static_cast<float*>(workspace);
    return launch_attention(d, as_stream(stream));
}

int qblora_rms_norm_fwd(const qblora_bf16* x, const qblora_bf16* residual, const qblora_bf16* w, int64_t T, int32_t d,
                        float eps, qblora_bf16* total, qblora_bf16* y, float* rstd, void* stream) {
    const int rc = check_norm(x, w, T, d);
    if (rc) return rc;
    if (T == 0) return QBLORA_OK;
    if (!y || (residual && !total)) return QBLORA_ERR_NULL;
    NormDesc a{x, residual, w, T, d, eps, total, y, rstd};
    return launch_rms_norm(a, as_stream(stream));
}

size_t qblora_rms_norm_bwd_workspace_bytes(int64_t T, int32_t d) {
    if (T <= 0 || d <= 0 || d > 16384) return 0;
    return (size_t)rms_norm_bwd_parts(T, d) * d * sizeof(float);
}

int qblora_rms_norm_bwd(const qblora_bf16* total, const qblora_bf16* w, const float* rstd, const qblora_bf16* dy,
                        const qblora_bf16* dtotal, int64_t T, int32_t d, qblora_bf16* dx, float* dw, void* workspace,
                        size_t workspace_bytes, void* stream) {
    const int rc = check_norm(total, w, T, d);
    if (rc) return rc;
    if (T && (!rstd || !dy || !dx)) return QBLORA_ERR_NULL;
    if (dw && T) {
        if (!workspace || workspace_bytes < qblora_rms_norm_bwd_workspace_bytes(T, d)) return QBLORA_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return QBLORA_ERR_SHAPE;
    }
    if (T == 0 && !dw) return QBLORA_OK;
    NormBackDesc a{total, w, rstd, dy, dtotal, T, d, dx, dw, dw ? static_cast<float*>(workspace) : nullptr, 0};
    return launch_rms_norm_bwd(a, as_stream(stream));
}

}  // extern "C"
