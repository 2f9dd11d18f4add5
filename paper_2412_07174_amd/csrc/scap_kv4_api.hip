// extern "C" entry points of the 4-bit key/value cache: argument validation and dispatch.  See include/scap.h.
#include <math.h>

#include "scap_kv4.hpp"
#include "scap_kv4_split.hpp"

using namespace scap;

namespace {

constexpr int64_t kMaxPages = (int64_t)1 << 24;
constexpr int64_t kMaxLayerBytes = ((int64_t)1 << 36) - 16;
constexpr int64_t kMaxSeqs = (int64_t)1 << 20;
constexpr int64_t kMaxNew = (int64_t)1 << 22;
constexpr int64_t kMaxRowTokens = kKv4MaxRange;
constexpr int64_t kMaxGroups = ((int64_t)1 << 23) - 1;  // workgroups of up to 512 threads: fewer than 2^32 threads
constexpr size_t kCounterBytes = (size_t)1 << 20;    // arrival counters at the start of a workspace

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// whether n words at a and m at b have one in common
bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + 4 * (uintptr_t)m && y < x + 4 * (uintptr_t)n;
}

int log2_of(int v) {
    for (int i = 0; i < 31; ++i)
        if (v == 1 << i) return i;
    return -1;
}

int check_cache(const scap_kv4_cache* c, bool refs) {
    if (!c || !c->pool || (refs && !c->refs)) return SCAP_ERR_NULL;
    if (scap_kv4_block_bytes(c->head_dim, c->page_tokens) == 0) return SCAP_ERR_SHAPE;
    if (c->pages < 1 || c->pages > kMaxPages || c->kv_heads < 1 || c->layers < 1) return SCAP_ERR_SHAPE;
    if ((int64_t)c->kv_heads * c->layers > 65536) return SCAP_ERR_SHAPE;
    // (pages lie at 32-bit offsets of 16 bytes in a layer)
    if (c->pages > kMaxLayerBytes / ((int64_t)c->kv_heads * kv4_block_bytes(c->head_dim, c->page_tokens))) return SCAP_ERR_SHAPE;
    if (!aligned(c->pool, 16) || !aligned(c->refs, 4)) return SCAP_ERR_ALIGN;
    return SCAP_OK;
}

Kv4Pool pool_of(const scap_kv4_cache& c) {
    return {static_cast<char*>(c.pool), c.refs, c.pages, c.kv_heads, c.head_dim, c.page_tokens, log2_of(c.page_tokens), c.layers};
}

int check_rows(const scap_kv4_cache& c, const int32_t* table, int64_t S, int64_t B) {
    if (!table) return SCAP_ERR_NULL;
    if (B < 1 || B > kMaxSeqs || S < 1 || S > kMaxRowTokens / c.page_tokens) return SCAP_ERR_SHAPE;
    if (B * ((S + 255) / 256) > kMaxGroups) return SCAP_ERR_SHAPE;
    return aligned(table, 4) ? SCAP_OK : SCAP_ERR_ALIGN;
}

int check_seqs(const scap_kv4_cache& c, int64_t layer, int dt, int64_t T, const int32_t* starts, const int32_t* table,
               int64_t S, const int32_t* lens, int64_t B) {
    if (!starts || !lens) return SCAP_ERR_NULL;
    if (dt != SCAP_F16 && dt != SCAP_BF16) return SCAP_ERR_DTYPE;
    if (layer < 0 || layer >= c.layers || T < 0 || T > kMaxNew) return SCAP_ERR_SHAPE;
    if (!aligned(starts, 4) || !aligned(lens, 4)) return SCAP_ERR_ALIGN;
    return check_rows(c, table, S, B);
}

int check_ws(const void* ws, size_t bytes, size_t need) {
    if (!ws) return SCAP_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return SCAP_ERR_ALIGN;
    return need == 0 || bytes < need ? SCAP_ERR_WORKSPACE : SCAP_OK;
}

size_t page_bytes_of(const scap_kv4_cache& c, int64_t B) {
    return kCounterBytes + align_up(4 * kv4_page_scratch_words(c.pages, B), 256);
}

// The page calls' scratch lies where attention keeps its partial results: both are dead when a call has ended.
int32_t* page_scratch(void* ws) { return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + kCounterBytes); }

bool attention_shape_ok(const scap_kv4_cache& c, int64_t B, int64_t T, int64_t heads) {
    return heads >= 1 && heads <= 65536 && heads % c.kv_heads == 0 && B >= 1 && B <= kMaxSeqs && T >= 0 && T <= kMaxNew &&
           T * (heads / c.kv_heads) < ((int64_t)1 << 30);
}

}  // namespace

extern "C" {

size_t scap_kv4_block_bytes(int32_t head_dim, int32_t page_tokens) {
    if (head_dim != 64 && head_dim != 128) return 0;
    if (page_tokens < 16 || page_tokens > 256 || log2_of(page_tokens) < 0) return 0;
    return (size_t)kv4_block_bytes(head_dim, page_tokens);
}

size_t scap_kv4_workspace_bytes(const scap_kv4_cache* cache, int64_t seqs, int64_t tokens, int64_t heads, int64_t max_new) {
    if (!cache || scap_kv4_block_bytes(cache->head_dim, cache->page_tokens) == 0) return 0;
    if (cache->pages < 1 || cache->pages > kMaxPages || cache->kv_heads < 1 || seqs < 1 || seqs > kMaxSeqs || max_new < 0) return 0;
    size_t need = page_bytes_of(*cache, seqs);
    if (heads != 0) {
        if (!attention_shape_ok(*cache, seqs, tokens, heads)) return 0;
        const Kv4AttnPlan p = plan_kv4_attention(cache->head_dim, cache->kv_heads, seqs, tokens,
                                                 (int)(heads / cache->kv_heads), max_new ? max_new : tokens);
        if (p.grid > kMaxGroups) return 0;
        const size_t attn = kCounterBytes + align_up(kv4_partial_bytes(cache->head_dim, cache->kv_heads, tokens, (int)(heads / cache->kv_heads), max_new ? max_new : tokens), 256);
        if (attn > need) need = attn;
    }
    return need;
}

int scap_kv4_append(const scap_kv4_cache* cache, int64_t layer, const void* k, int64_t k_stride_token, int64_t k_stride_head,
                    const void* v, int64_t v_stride_token, int64_t v_stride_head, int dt, int64_t T, const int32_t* starts,
                    const int32_t* table, int64_t S, const int32_t* lens, int64_t B, void* stream) {
    int rc = check_cache(cache, false);
    if (rc == SCAP_OK && (!k || !v) && T != 0) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_seqs(*cache, layer, dt, T, starts, table, S, lens, B);
    if (rc != SCAP_OK) return rc;
    if (!aligned(k, 2) || !aligned(v, 2)) return SCAP_ERR_ALIGN;
    if (T == 0) return SCAP_OK;
    Kv4TokensArgs a{};
    a.p = pool_of(*cache);
    a.s = {starts, table, lens, (int)B, (int)S, (int)T};
    a.layer = (int)layer;
    a.dt = dt;
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.k_st = k_stride_token, a.k_sh = k_stride_head, a.v_st = v_stride_token, a.v_sh = v_stride_head;
    return launch_kv4_append(a, static_cast<hipStream_t>(stream));
}

int scap_kv4_read(const scap_kv4_cache* cache, int64_t layer, void* k_out, void* v_out, int dt, int64_t T,
                  const int32_t* starts, const int32_t* table, int64_t S, const int32_t* lens, int64_t B, void* stream) {
    int rc = check_cache(cache, false);
    if (rc == SCAP_OK && (!k_out || !v_out) && T != 0) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_seqs(*cache, layer, dt, T, starts, table, S, lens, B);
    if (rc != SCAP_OK) return rc;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return SCAP_ERR_ALIGN;
    if (T == 0) return SCAP_OK;
    Kv4TokensArgs a{};
    a.p = pool_of(*cache);
    a.s = {starts, table, lens, (int)B, (int)S, (int)T};
    a.layer = (int)layer;
    a.dt = dt;
    a.k_out = static_cast<uint16_t*>(k_out);
    a.v_out = static_cast<uint16_t*>(v_out);
    return launch_kv4_read(a, static_cast<hipStream_t>(stream));
}

int scap_kv4_attention(const scap_kv4_cache* cache, int64_t layer, const void* q, int64_t q_stride_token,
                       int64_t q_stride_head, int dt, int64_t heads, int64_t T, const int32_t* starts, const int32_t* table,
                       int64_t S, const int32_t* lens, int64_t B, int64_t max_new, float scale, int causal, int64_t window,
                       void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache, false);
    if (rc == SCAP_OK && (!q || !out) && T != 0) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_seqs(*cache, layer, dt, T, starts, table, S, lens, B);
    if (rc != SCAP_OK) return rc;
    if (!attention_shape_ok(*cache, B, T, heads) || max_new < 0 || window < 0 || window > ((int64_t)1 << 30)) return SCAP_ERR_SHAPE;
    if (!(scale > 0.f) || !isfinite(scale)) return SCAP_ERR_VALUE;
    if (window > 0 && !causal) return SCAP_ERR_VALUE;
    if (!aligned(q, 2) || !aligned(out, 16) || !aligned(lse, 4)) return SCAP_ERR_ALIGN;
    const int G = (int)(heads / cache->kv_heads);
    const Kv4AttnPlan plan = plan_kv4_attention(cache->head_dim, cache->kv_heads, B, T, G, max_new ? max_new : T);
    if (plan.grid > kMaxGroups) return SCAP_ERR_SHAPE;
    static_assert(3 * 65536 * 4 <= kCounterBytes && (1024 + 2 * 1024) * 4 <= kCounterBytes, "(places + 2) * kv_heads counters");
    rc = check_ws(workspace, workspace_bytes, scap_kv4_workspace_bytes(cache, B, T, heads, max_new));
    if (rc != SCAP_OK) return rc;
    if (T == 0) return SCAP_OK;
    Kv4AttnArgs a{};
    a.p = pool_of(*cache);
    a.s = {starts, table, lens, (int)B, (int)S, (int)T};
    a.layer = (int)layer;
    a.dt = dt;
    a.q = static_cast<const uint16_t*>(q);
    a.q_st = q_stride_token, a.q_sh = q_stride_head;
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.H = (int)heads;
    a.G = G;
    a.scale = scale * 1.4426950408889634f;
    a.causal = causal != 0;
    a.window = (int)window;
    a.inv_G = 1.0 / G;
    a.places = plan.places;
    a.min_chunk = plan.min_chunk;
    a.counters = static_cast<int32_t*>(workspace);
    a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
    a.slot_floats = plan.slot_floats;
    a.slot_rows = plan.slot_rows;
    const size_t room = workspace_bytes - kCounterBytes;
    a.partial_bytes = room < 0xFFFFFFFFu ? (uint32_t)room : 0xFFFFFFFFu;
    return launch_kv4_attention(a, plan, static_cast<hipStream_t>(stream));
}

int scap_kv4_reserve(const scap_kv4_cache* cache, int32_t* table, int64_t S, int64_t B, const int32_t* old_lens,
                     const int32_t* new_lens, int32_t* info, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache, true);
    if (rc == SCAP_OK && (!old_lens || !new_lens || !info)) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_rows(*cache, table, S, B);
    if (rc != SCAP_OK) return rc;
    if (B > kKv4MaxReserve) return SCAP_ERR_SHAPE;
    if (!aligned(old_lens, 4) || !aligned(new_lens, 4) || !aligned(info, 4)) return SCAP_ERR_ALIGN;
    rc = check_ws(workspace, workspace_bytes, page_bytes_of(*cache, B));
    if (rc != SCAP_OK) return rc;
    return launch_kv4_reserve(pool_of(*cache), table, (int)S, (int)B, old_lens, new_lens, info, page_scratch(workspace),
                              static_cast<hipStream_t>(stream));
}

int scap_kv4_fork(const scap_kv4_cache* cache, const int32_t* table, const int32_t* lens, int64_t B_in, const int32_t* parents,
                  int64_t B_out, int32_t* table_out, int32_t* lens_out, int64_t S, void* stream) {
    int rc = check_cache(cache, true);
    if (rc == SCAP_OK && (!lens || !parents || !lens_out)) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_rows(*cache, table, S, B_in);
    if (rc == SCAP_OK) rc = check_rows(*cache, table_out, S, B_out);
    if (rc != SCAP_OK) return rc;
    if (!aligned(lens, 4) || !aligned(parents, 4) || !aligned(lens_out, 4)) return SCAP_ERR_ALIGN;
    // a row's length and pages are written while other workgroups still read theirs
    const int64_t in = B_in * S, out = B_out * S;
    if (overlap(table_out, out, table, in) || overlap(table_out, out, lens, B_in) || overlap(table_out, out, parents, B_out) ||
        overlap(lens_out, B_out, table, in) || overlap(lens_out, B_out, lens, B_in) || overlap(lens_out, B_out, parents, B_out) ||
        overlap(table_out, out, lens_out, B_out))
        return SCAP_ERR_VALUE;
    return launch_kv4_fork(pool_of(*cache), table, lens, (int)B_in, parents, (int)B_out, table_out, lens_out, (int)S,
                           static_cast<hipStream_t>(stream));
}

int scap_kv4_free(const scap_kv4_cache* cache, int32_t* table, int64_t S, int64_t B, const int32_t* keep_from,
                  const int32_t* keep_to, void* stream) {
    int rc = check_cache(cache, true);
    if (rc == SCAP_OK) rc = check_rows(*cache, table, S, B);
    if (rc != SCAP_OK) return rc;
    if (!aligned(keep_from, 4) || !aligned(keep_to, 4)) return SCAP_ERR_ALIGN;
    return launch_kv4_free(pool_of(*cache), table, (int)S, (int)B, keep_from, keep_to, static_cast<hipStream_t>(stream));
}

int scap_kv4_compact(const scap_kv4_cache* cache, const int32_t* table, int64_t S, int64_t B, int32_t* table_out,
                     int32_t* refs_out, int32_t* info, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache, true);
    if (rc == SCAP_OK && (!table_out || !refs_out || !info)) rc = SCAP_ERR_NULL;
    if (rc == SCAP_OK) rc = check_rows(*cache, table, S, B);
    if (rc != SCAP_OK) return rc;
    if (!aligned(table_out, 4) || !aligned(refs_out, 4) || !aligned(info, 4)) return SCAP_ERR_ALIGN;
    rc = check_ws(workspace, workspace_bytes, page_bytes_of(*cache, B));
    if (rc != SCAP_OK) return rc;
    return launch_kv4_compact(pool_of(*cache), table, (int)S, (int)B, table_out, refs_out, info, page_scratch(workspace),
                              static_cast<hipStream_t>(stream));
}

int scap_kv4_copy_pages(const scap_kv4_cache* from, const scap_kv4_cache* to, const int32_t* src, const int32_t* dst,
                        int64_t n, void* stream) {
    int rc = check_cache(from, false);
    if (rc == SCAP_OK) rc = check_cache(to, false);
    if (rc == SCAP_OK && (!src || !dst) && n != 0) rc = SCAP_ERR_NULL;
    if (rc != SCAP_OK) return rc;
    if (from->kv_heads != to->kv_heads || from->head_dim != to->head_dim || from->page_tokens != to->page_tokens ||
        from->layers != to->layers || n < 0 || n > kMaxPages)
        return SCAP_ERR_SHAPE;
    if (!aligned(src, 4) || !aligned(dst, 4)) return SCAP_ERR_ALIGN;
    if (n == 0) return SCAP_OK;
    return launch_kv4_copy_pages(pool_of(*from), pool_of(*to), src, dst, n, static_cast<hipStream_t>(stream));
}

int scap_kv4_call(int what, const int64_t* w) {
    if (!w) return SCAP_ERR_NULL;
    static constexpr int kWords[] = {16, 12, 22, 10, 10, 7, 10};
    const int n = what >> 8;
    what &= 0xFF;
    if (n < 0 || what > SCAP_KV4_COMPACT || (n != 0 && n != kWords[what])) return SCAP_ERR_VALUE;
    const auto ptr = [&](int i) { return reinterpret_cast<void*>(static_cast<uintptr_t>(w[i])); };
    const auto ints = [&](int i) { return static_cast<int32_t*>(ptr(i)); };
    const auto cache = static_cast<const scap_kv4_cache*>(ptr(0));
    switch (what) {
        case SCAP_KV4_APPEND:
            return scap_kv4_append(cache, w[1], ptr(2), w[3], w[4], ptr(5), w[6], w[7], (int)w[8], w[9], ints(10), ints(11), w[12],
                                   ints(13), w[14], ptr(15));
        case SCAP_KV4_READ:
            return scap_kv4_read(cache, w[1], ptr(2), ptr(3), (int)w[4], w[5], ints(6), ints(7), w[8], ints(9), w[10], ptr(11));
        case SCAP_KV4_ATTENTION: {
            const uint32_t bits = (uint32_t)w[14];
            float scale;
            static_assert(sizeof(scale) == sizeof(bits), "");
            __builtin_memcpy(&scale, &bits, sizeof(scale));
            return scap_kv4_attention(cache, w[1], ptr(2), w[3], w[4], (int)w[5], w[6], w[7], ints(8), ints(9), w[10], ints(11), w[12],
                                      w[13], scale, (int)w[15], w[16], ptr(17), static_cast<float*>(ptr(18)), ptr(19),
                                      (size_t)w[20], ptr(21));
        }
        case SCAP_KV4_RESERVE:
            return scap_kv4_reserve(cache, ints(1), w[2], w[3], ints(4), ints(5), ints(6), ptr(7), (size_t)w[8], ptr(9));
        case SCAP_KV4_FORK:
            return scap_kv4_fork(cache, ints(1), ints(2), w[3], ints(4), w[5], ints(6), ints(7), w[8], ptr(9));
        case SCAP_KV4_FREE: return scap_kv4_free(cache, ints(1), w[2], w[3], ints(4), ints(5), ptr(6));
        case SCAP_KV4_COMPACT:
            return scap_kv4_compact(cache, ints(1), w[2], w[3], ints(4), ints(5), ints(6), ptr(7), (size_t)w[8], ptr(9));
    }
    return SCAP_ERR_VALUE;
}

}  // extern "C"
