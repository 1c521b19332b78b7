// The serving calls of include/agq.h: argument checks on the host (before any HIP call), then the launchers.
#include "../../include/agq.h"
#include <initializer_list>
#include "agq_internal.h"

namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int64_t kMaxIndex = 0x7FFFFFFF;
constexpr int64_t kMaxHeads = 65536;
constexpr int64_t kMaxRow = (int64_t)1 << 24;
constexpr int64_t kMaxGroups = (int64_t)1 << 24;      // workgroups of 256: a launch has less than 2^32 threads in a dimension

inline int hip_status(int err) { return err == 0 ? AGQ_OK : AGQ_EHIP; }
inline bool aligned(const void *p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool ints_ok(const void *p) { return aligned(p, 4); }
inline bool page_ok(int64_t page) { return page == 16 || page == 32 || page == 64 || page == 128; }
inline bool count_ok(int64_t n, int64_t most) { return n >= 0 && n <= most; }
// a fp16 tensor [tokens, heads, D]
inline bool tensor_ok(const void *p, int64_t ld, int64_t heads, int64_t D) {
    return aligned(p, 16) && ld >= heads * D && ld % 8 == 0 && ld <= kMaxTokens;
}
// gains: one row for all heads (ld = 0) or one for each
inline bool gain_ok(const void *p, int64_t ld, int64_t D) { return aligned(p, 16) && (ld == 0 || (ld >= D && ld % 8 == 0 && ld <= kMaxTokens)); }
inline bool heads_ok(int64_t Hq, int64_t Hkv, int64_t D) {
    return (D == 64 || D == 128) && Hkv >= 1 && Hkv <= kMaxHeads && Hq >= Hkv && Hq <= kMaxHeads && Hq % Hkv == 0;
}
inline bool cache_ok(const agq_kv_cache *c) {
    return c && page_ok(c->page) && (c->D == 64 || c->D == 128) && c->Hkv >= 1 && c->Hkv <= kMaxHeads && c->n_pages >= 1 &&
           c->n_pages <= kMaxIndex / c->page && aligned(c->k, 16) && aligned(c->v, 16) && c->k_exp && c->v_exp;
}
// with it the largest and smallest scores that fp16 queries and keys, or codes of exponents -64 to 64, can make are normal fp32 numbers
inline bool scale_ok(float s) { return s >= 0x1p-60f && s <= 0x1p24f; }
inline bool apart(const void *a, size_t an, const void *b, size_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x + an <= y || y + bn <= x;
}

}  // namespace

int agq_kv_map(const int32_t *kv_len, const int32_t *n_new, int64_t B, int64_t page, int32_t *block_table, int64_t max_pages,
               int32_t *free_ring, int64_t n_pages, const int32_t *free_state, int64_t T, int32_t *kv_len_out, int32_t *cu_new,
               int32_t *pos, int32_t *slot, int32_t *free_state_out, int32_t *status, void *stream) {
    if (!count_ok(B, (int64_t)1 << 20) || !count_ok(T, kMaxTokens) || !page_ok(page)) return AGQ_EINVAL;
    if (max_pages < 1 || max_pages > kMaxIndex / page || n_pages < 1 || n_pages > kMaxIndex / page) return AGQ_EINVAL;
    if (!ints_ok(free_ring) || !ints_ok(free_state) || !ints_ok(free_state_out) || !ints_ok(cu_new) || !ints_ok(status)) return AGQ_EINVAL;
    if (B > 0 && (!ints_ok(kv_len) || !ints_ok(n_new) || !ints_ok(block_table) || !ints_ok(kv_len_out))) return AGQ_EINVAL;
    if (T > 0 && (!ints_ok(pos) || !ints_ok(slot))) return AGQ_EINVAL;
    if (!apart(free_state, 8, free_state_out, 8) || (B > 0 && !apart(kv_len, 4 * (size_t)B, kv_len_out, 4 * (size_t)B))) return AGQ_EINVAL;
    return hip_status(agq_launch_kv_map(kv_len, n_new, B, (int)page, block_table, max_pages, free_ring, n_pages, free_state, T, kv_len_out,
                                        cu_new, pos, slot, free_state_out, status, stream));
}

// the appends: norm says that the heads of q and k are normalised, with gains g_q and g_k
static int append(bool norm, const agq_kv_cache *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t T, const int32_t *slot,
                  const void *q, int64_t ldq, int64_t Hq, const void *g_q, int64_t ldgq, const void *g_k, int64_t ldgk, double eps,
                  const int32_t *pos, const float *rope_cos, const float *rope_sin, int64_t P, void *q_out, int64_t ldqo, void *k_out,
                  int64_t ldko, void *stream) {
    if (!cache_ok(cache) || !count_ok(T, kMaxTokens)) return AGQ_EINVAL;
    const int64_t D = cache->D, Hkv = cache->Hkv;
    if (Hq < 0 || Hq > kMaxHeads) return AGQ_EINVAL;
    if (norm && !(eps >= 0.0)) return AGQ_EINVAL;
    if (T == 0) return AGQ_OK;                                            // tensors of no tokens have no addresses
    const bool rope = rope_cos || rope_sin || pos;
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (Hq > 0)) return AGQ_EINVAL;
    if (!rope && !norm && (q || k_out)) return AGQ_EINVAL;
    if (rope && (P < 1 || P > kMaxIndex || !aligned(rope_cos, 16) || !aligned(rope_sin, 16))) return AGQ_EINVAL;
    if (norm && ((g_q != nullptr) != (q != nullptr) || !gain_ok(g_k, ldgk, D) || (g_q && !gain_ok(g_q, ldgq, D)))) return AGQ_EINVAL;
    // workgroups and work items are counted in 31 bits
    if (T * (D / 16) > kMaxIndex / (Hq > 2 * Hkv ? Hq : 2 * Hkv) - 4096) return AGQ_EINVAL;
    if (!ints_ok(slot) || (rope && !ints_ok(pos)) || !tensor_ok(k, ldk, Hkv, D) || !tensor_ok(v, ldv, Hkv, D)) return AGQ_EINVAL;
    if (q && (!tensor_ok(q, ldq, Hq, D) || !tensor_ok(q_out, ldqo, Hq, D))) return AGQ_EINVAL;
    if (k_out && !tensor_ok(k_out, ldko, Hkv, D)) return AGQ_EINVAL;
    const AgqKvAppend a = {cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, Hkv, D, (int)cache->page, q, k, v, q_out, k_out,
                           ldq, ldk, ldv, ldqo, ldko, T, Hq, P, pos, slot, rope_cos, rope_sin, g_q, g_k, ldgq, ldgk, eps};
    return hip_status(agq_launch_kv_append(a, stream));
}

int agq_kv_append(const agq_kv_cache *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t T, const int32_t *slot,
                  const void *q, int64_t ldq, int64_t Hq, const int32_t *pos, const float *rope_cos, const float *rope_sin, int64_t P,
                  void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *stream) {
    return append(false, cache, k, ldk, v, ldv, T, slot, q, ldq, Hq, nullptr, 0, nullptr, 0, 0.0, pos, rope_cos, rope_sin, P, q_out, ldqo, k_out,
                  ldko, stream);
}

int agq_kv_append_norm(const agq_kv_cache *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t T, const int32_t *slot,
                       const void *q, int64_t ldq, int64_t Hq, const void *g_q, int64_t ldgq, const void *g_k, int64_t ldgk, double eps,
                       const int32_t *pos, const float *rope_cos, const float *rope_sin, int64_t P, void *q_out, int64_t ldqo, void *k_out,
                       int64_t ldko, void *stream) {
    return append(true, cache, k, ldk, v, ldv, T, slot, q, ldq, Hq, g_q, ldgq, g_k, ldgk, eps, pos, rope_cos, rope_sin, P, q_out, ldqo, k_out,
                  ldko, stream);
}

int agq_qk_norm_rope(const void *q, int64_t ldq, int64_t Hq, const void *k, int64_t ldk, int64_t Hkv, int64_t T, int64_t D, const void *g_q,
                     int64_t ldgq, const void *g_k, int64_t ldgk, double eps, const int32_t *pos, const float *rope_cos, const float *rope_sin,
                     int64_t P, void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *stream) {
    if (!count_ok(T, kMaxTokens) || !count_ok(Hq, kMaxHeads) || !count_ok(Hkv, kMaxHeads) || (D != 64 && D != 128) || !(eps >= 0.0)) return AGQ_EINVAL;
    if (T == 0) return AGQ_OK;                                            // tensors of no tokens have no addresses
    const bool rope = rope_cos || rope_sin || pos;
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (Hq > 0) || (k != nullptr) != (k_out != nullptr) || (k != nullptr) != (Hkv > 0))
        return AGQ_EINVAL;
    if ((!q && !k) || (g_q && !q) || (g_k && !k) || (!rope && !g_q && !g_k)) return AGQ_EINVAL;
    if (T * (D / 16) > kMaxIndex / (Hq + Hkv)) return AGQ_EINVAL;         // work items are counted in 31 bits
    if (rope && (P < 1 || P > kMaxIndex || !aligned(rope_cos, 16) || !aligned(rope_sin, 16) || !ints_ok(pos))) return AGQ_EINVAL;
    if (q && (!tensor_ok(q, ldq, Hq, D) || !tensor_ok(q_out, ldqo, Hq, D))) return AGQ_EINVAL;
    if (k && (!tensor_ok(k, ldk, Hkv, D) || !tensor_ok(k_out, ldko, Hkv, D))) return AGQ_EINVAL;
    if ((g_q && !gain_ok(g_q, ldgq, D)) || (g_k && !gain_ok(g_k, ldgk, D))) return AGQ_EINVAL;
    const AgqQkNormRope a = {q, k, g_q, g_k, q_out, k_out, ldq, ldk, ldgq, ldgk, ldqo, ldko, T, Hq, Hkv, D, P, pos, rope_cos, rope_sin, eps};
    return hip_status(agq_launch_qk_norm_rope(a, stream));
}

size_t agq_attn_packed_workspace_bytes(int64_t Tq, int64_t Hq, int64_t Tk, int64_t Hkv, int64_t D, int64_t B) {
    if (!heads_ok(Hq, Hkv, D) || !count_ok(Tq, kMaxTokens) || !count_ok(Tk, kMaxTokens) || !count_ok(B, (int64_t)1 << 20)) return 0;
    const AgqPackedSplit s = agq_packed_split(Tq, Tk, B, Hq, D);
    return s.splits == 1 ? 0 : (size_t)s.splits * (size_t)Tq * (size_t)Hq * (size_t)(D * 4 + 8);
}

int agq_attn_packed(const void *q, int64_t ldq, int64_t Tq, int64_t Hq, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t Tk,
                    int64_t Hkv, int64_t D, const int32_t *cu_q, const int32_t *cu_k, int64_t B, int causal, float scale, void *o,
                    int64_t ldo, void *workspace, size_t workspace_bytes, void *stream) {
    if (!heads_ok(Hq, Hkv, D) || !count_ok(Tq, kMaxTokens) || !count_ok(Tk, kMaxTokens) || !count_ok(B, (int64_t)1 << 20) || !scale_ok(scale))
        return AGQ_EINVAL;
    if (agq_packed_tiles(Tq, B) * Hq >= kMaxGroups) return AGQ_EINVAL;
    if (ldk > kMaxRow || ldv > kMaxRow) return AGQ_EINVAL;                // 32 rows are reached by 32-bit offsets
    if (Tq == 0 || B == 0) return AGQ_OK;
    if (!ints_ok(cu_q) || !ints_ok(cu_k) || !tensor_ok(q, ldq, Hq, D) || !tensor_ok(o, ldo, Hq, D)) return AGQ_EINVAL;
    if (Tk > 0 && (!tensor_ok(k, ldk, Hkv, D) || !tensor_ok(v, ldv, Hkv, D))) return AGQ_EINVAL;
    const AgqAttnPacked a = {q, k, v, o, ldq, ldk, ldv, ldo, Tq, Tk, Hq, Hkv, D, B, cu_q, cu_k, causal != 0, scale};
    const size_t need = agq_attn_packed_workspace_bytes(Tq, Hq, Tk, Hkv, D, B);
    if (need > 0) {
        if (!aligned(workspace, 16)) return AGQ_EINVAL;
        if (workspace_bytes < need) return AGQ_ESIZE;
    }
    return hip_status(agq_launch_attn_packed(a, agq_packed_split(Tq, Tk, B, Hq, D), workspace, stream));
}

size_t agq_attn_kv_workspace_bytes(int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t B, int64_t max_q, int64_t max_kv) {
    if (!heads_ok(Hq, Hkv, D) || !count_ok(T, kMaxTokens) || !count_ok(B, 65535) || !count_ok(max_q, kMaxTokens) || !count_ok(max_kv, kMaxTokens))
        return 0;
    const AgqKvSplit s = agq_kv_split(B, Hq, Hkv, max_q, max_kv);
    return s.splits == 1 ? 0 : (size_t)s.splits * (size_t)T * (size_t)Hq * (size_t)(D * 4 + 8);
}

int agq_attn_kv(const agq_kv_cache *cache, const void *q, int64_t ldq, int64_t T, int64_t Hq, const int32_t *cu_q, const int32_t *kv_len,
                int64_t B, const int32_t *block_table, int64_t max_pages, int64_t max_q, int64_t max_kv, float scale, void *o, int64_t ldo,
                void *workspace, size_t workspace_bytes, void *stream) {
    if (!cache_ok(cache) || !heads_ok(Hq, cache->Hkv, cache->D) || Hq / cache->Hkv > 1024) return AGQ_EINVAL;
    if (!count_ok(T, kMaxTokens) || !count_ok(B, 65535) || !count_ok(max_q, kMaxTokens) || !count_ok(max_kv, kMaxTokens) || !scale_ok(scale))
        return AGQ_EINVAL;
    if (max_pages < 1 || max_pages > kMaxTokens / cache->page) return AGQ_EINVAL;   // keys are counted in 31 bits, with a chunk or two to spare
    const AgqKvSplit s = agq_kv_split(B, Hq, cache->Hkv, max_q, max_kv);
    if (B * cache->Hkv * s.row_tiles > kMaxIndex / s.splits) return AGQ_EINVAL;      // workgroups
    if (T == 0 || B == 0) return AGQ_OK;
    if (!ints_ok(cu_q) || !ints_ok(kv_len) || !ints_ok(block_table) || !tensor_ok(q, ldq, Hq, cache->D) || !tensor_ok(o, ldo, Hq, cache->D))
        return AGQ_EINVAL;
    const size_t need = agq_attn_kv_workspace_bytes(T, Hq, cache->Hkv, cache->D, B, max_q, max_kv);
    if (need > 0) {
        if (!aligned(workspace, 16)) return AGQ_EINVAL;
        if (workspace_bytes < need) return AGQ_ESIZE;
    }
    const AgqAttnKv a = {cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, cache->Hkv, cache->D, (int)cache->page, q, o, ldq, ldo,
                         T, Hq, B, max_pages, max_q, cu_q, kv_len, block_table, scale};
    return hip_status(agq_launch_attn_kv(a, s, workspace, stream));
}

static_assert(AGQ_KV_MAX_FORK == AGQ_KV_MAX_B, "the kernels hold that many requests' sums");
struct Ints {
    const int32_t *p;
    int64_t n;
};
// what agq_kv_fork and agq_kv_compact have in common, and what they read and write beside it: workgroups write while others read
static bool pages_ok(const AgqKvPages &p, std::initializer_list<Ints> more_in, std::initializer_list<Ints> more_out) {
    if (!count_ok(p.B, AGQ_KV_MAX_FORK) || !page_ok(p.page)) return false;
    if (p.max_pages < 1 || p.max_pages > kMaxIndex / p.page || p.n_pages < 1 || p.n_pages > kMaxIndex / p.page) return false;
    Ints all[16];
    int n = 0, n_out = 0;
    bool ok = true;
    auto take = [&](const Ints &t) {                                      // tensors of no values have no addresses
        ok &= t.n == 0 || ints_ok(t.p);
        if (t.n > 0) all[n++] = t;
    };
    const int64_t entries = p.B * p.max_pages;
    for (const Ints &t : {Ints{p.ring, p.n_pages}, {p.kv_len_out, p.B}, {p.table_out, entries}, {p.shared_out, p.n_pages}, {p.free_out, 2}, {p.status, 1}}) take(t);
    for (const Ints &t : more_out) take(t);
    n_out = n;
    for (const Ints &t : {Ints{p.kv_len, p.B}, {p.table, entries}, {p.shared, p.n_pages}, {p.free_in, 2}}) take(t);
    for (const Ints &t : more_in) take(t);
    for (int i = 0; i < n_out; ++i)
        for (int j = i + 1; j < n; ++j) ok &= apart(all[i].p, 4 * (size_t)all[i].n, all[j].p, 4 * (size_t)all[j].n);
    return ok;
}

int agq_kv_fork(const int32_t *kv_len, const int32_t *parent, int64_t B, int64_t page, const int32_t *block_table, int64_t max_pages,
                const int32_t *shared, int32_t *free_ring, int64_t n_pages, const int32_t *free_state, int32_t *kv_len_out,
                int32_t *block_table_out, int32_t *shared_out, int32_t *copy_src, int32_t *copy_dst, int32_t *free_state_out, int32_t *status,
                void *stream) {
    const AgqKvPages p = {kv_len, block_table, shared, free_state, free_ring, kv_len_out, block_table_out, shared_out, free_state_out, status, B, page,
                          max_pages, n_pages};
    if (!pages_ok(p, {{parent, B}}, {{copy_src, B}, {copy_dst, B}})) return AGQ_EINVAL;
    return hip_status(agq_launch_kv_fork(p, parent, copy_src, copy_dst, stream));
}

size_t agq_kv_moves_ints(int64_t N, int64_t B, int64_t page) {
    if (!count_ok(N, kMaxTokens - 1) || !count_ok(B, AGQ_KV_MAX_FORK) || !page_ok(page)) return 0;
    return (size_t)(4 + 4 * agq_kv_new_pages(N, B, page) + AGQ_KV_CHECKS);
}

int agq_kv_compact(const int32_t *kv_len, const int32_t *stay, const int32_t *cu_keep, const int32_t *keep, int64_t N, int64_t B, int64_t page,
                   const int32_t *block_table, int64_t max_pages, const int32_t *shared, int32_t *free_ring, int64_t n_pages,
                   const int32_t *free_state, int32_t *kv_len_out, int32_t *block_table_out, int32_t *shared_out, int32_t *moves,
                   int32_t *free_state_out, int32_t *status, void *stream) {
    const AgqKvPages p = {kv_len, block_table, shared, free_state, free_ring, kv_len_out, block_table_out, shared_out, free_state_out, status, B, page,
                          max_pages, n_pages};
    const int64_t n_moves = (int64_t)agq_kv_moves_ints(N, B, page);
    if (!count_ok(N, kMaxTokens - 1) || !aligned(moves, 16)) return AGQ_EINVAL;
    if (!pages_ok(p, {{stay, B}, {cu_keep, B + 1}, {keep, N}}, {{moves, n_moves}})) return AGQ_EINVAL;
    return hip_status(agq_launch_kv_compact(p, stay, cu_keep, keep, N, moves, stream));
}

// the caches of all layers: one shape
static bool layers_ok(const agq_kv_cache *c, int n) {
    if (n < 0 || n > 65536 || (n > 0 && !c)) return false;
    for (int i = 0; i < n; ++i)
        if (!cache_ok(c + i) || c[i].n_pages != c[0].n_pages || c[i].Hkv != c[0].Hkv || c[i].D != c[0].D || c[i].page != c[0].page) return false;
    return true;
}
// launch(shape, layers, count) for as many layers as a launch takes, one after the other
template <class F>
static int over_layers(const agq_kv_cache *c, int n, F launch) {
    for (int i = 0; i < n; i += AGQ_KV_LAYERS) {
        const int m = n - i < AGQ_KV_LAYERS ? n - i : AGQ_KV_LAYERS;
        AgqKvLayer layers[AGQ_KV_LAYERS];
        for (int l = 0; l < m; ++l) layers[l] = {c[i + l].k, c[i + l].v, c[i + l].k_exp, c[i + l].v_exp};
        if (const int err = launch(AgqKvShape{c->n_pages, c->Hkv, c->D, c->page}, layers, m)) return hip_status(err);
    }
    return AGQ_OK;
}

int agq_kv_copy_pages(const agq_kv_cache *caches, int n_caches, const int32_t *src, const int32_t *dst, int64_t n, void *stream) {
    if (!layers_ok(caches, n_caches) || !count_ok(n, (int64_t)1 << 20)) return AGQ_EINVAL;
    if (n == 0 || n_caches == 0) return AGQ_OK;
    if (!ints_ok(src) || !ints_ok(dst)) return AGQ_EINVAL;
    return over_layers(caches, n_caches,
                       [&](const AgqKvShape &s, const AgqKvLayer *l, int m) { return agq_launch_kv_copy_pages(s, l, m, src, dst, n, stream); });
}

int agq_kv_move(const agq_kv_cache *caches, int n_caches, const int32_t *moves, const int32_t *block_table, int64_t max_pages, const int32_t *stay,
                const int32_t *cu_keep, const int32_t *keep, int64_t N, int64_t B, void *stream) {
    if (!layers_ok(caches, n_caches) || !count_ok(N, kMaxTokens - 1) || !count_ok(B, AGQ_KV_MAX_FORK)) return AGQ_EINVAL;
    if (n_caches > 0 && (max_pages < 1 || max_pages > kMaxIndex / caches->page)) return AGQ_EINVAL;
    if (B == 0 || n_caches == 0) return AGQ_OK;
    if (!aligned(moves, 16) || !ints_ok(block_table) || !ints_ok(stay) || !ints_ok(cu_keep) || (N > 0 && !ints_ok(keep))) return AGQ_EINVAL;
    return over_layers(caches, n_caches, [&](const AgqKvShape &s, const AgqKvLayer *l, int m) {
        return agq_launch_kv_move(s, l, m, moves, block_table, max_pages, stay, cu_keep, keep, N, B, stream);
    });
}

size_t agq_logprobs_workspace_bytes(int64_t T, int64_t V, int kind, int64_t n_top) {
    if (!count_ok(T, (int64_t)1 << 22) || V < 1 || V > kMaxRow || (kind != AGQ_LOGITS_F16 && kind != AGQ_LOGITS_F32)) return 0;
    if (n_top < 0 || n_top > AGQ_MAX_TOP || n_top > V) return 0;
    return agq_logprobs_workspace(T, V, kind, n_top);
}

int agq_logprobs(const void *logits, int kind, int64_t T, int64_t V, int64_t ld, float scale, const int32_t *tokens, int64_t n_top, float *logprob,
                 float *entropy, int32_t *top_idx, float *top_logprob, void *workspace, size_t workspace_bytes, void *stream) {
    if (!count_ok(T, (int64_t)1 << 22) || V < 1 || V > kMaxRow || (kind != AGQ_LOGITS_F16 && kind != AGQ_LOGITS_F32)) return AGQ_EINVAL;
    if (n_top < 0 || n_top > AGQ_MAX_TOP || n_top > V || ld < V || ld > kMaxTokens) return AGQ_EINVAL;
    if (!(scale >= 0x1p-24f && scale <= 0x1p24f)) return AGQ_EINVAL;
    if (T == 0) return AGQ_OK;                                            // tensors of no rows have no addresses
    if ((tokens != nullptr) != (logprob != nullptr) || (n_top > 0 ? !top_idx || !top_logprob : top_idx || top_logprob)) return AGQ_EINVAL;
    if (!aligned(logits, kind == AGQ_LOGITS_F32 ? 4 : 2) || (tokens && (!ints_ok(tokens) || !ints_ok(logprob)))) return AGQ_EINVAL;
    if ((entropy && !ints_ok(entropy)) || (n_top > 0 && (!ints_ok(top_idx) || !ints_ok(top_logprob)))) return AGQ_EINVAL;
    const size_t need = agq_logprobs_workspace_bytes(T, V, kind, n_top);
    if (need > 0) {
        if (!aligned(workspace, 16)) return AGQ_EINVAL;
        if (workspace_bytes < need) return AGQ_ESIZE;
    }
    const AgqLogprobs a = {logits, kind, T, V, ld, n_top, scale, tokens, logprob, entropy, top_logprob, top_idx};
    return hip_status(agq_launch_logprobs(a, workspace, stream));
}
