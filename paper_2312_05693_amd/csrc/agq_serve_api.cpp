// The serving calls of include/agq.h: argument checks on the host (before any HIP call), then the launchers.
#include "../../include/agq.h"
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

int agq_kv_append(const agq_kv_cache *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, int64_t T, const int32_t *slot,
                  const void *q, int64_t ldq, int64_t Hq, const int32_t *pos, const float *rope_cos, const float *rope_sin, int64_t P,
                  void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *stream) {
    if (!cache_ok(cache) || !count_ok(T, kMaxTokens)) return AGQ_EINVAL;
    const int64_t D = cache->D, Hkv = cache->Hkv;
    if (Hq < 0 || Hq > kMaxHeads) return AGQ_EINVAL;
    if (T == 0) return AGQ_OK;                                            // tensors of no tokens have no addresses
    const bool rope = rope_cos || rope_sin || pos;
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (Hq > 0)) return AGQ_EINVAL;
    if (!rope && (q || k_out)) return AGQ_EINVAL;
    if (rope && (P < 1 || P > kMaxIndex || !aligned(rope_cos, 16) || !aligned(rope_sin, 16))) return AGQ_EINVAL;
    // workgroups and work items are counted in 31 bits
    if (T * (D / 16) > kMaxIndex / (Hq > 2 * Hkv ? Hq : 2 * Hkv) - 4096) return AGQ_EINVAL;
    if (!ints_ok(slot) || (rope && !ints_ok(pos)) || !tensor_ok(k, ldk, Hkv, D) || !tensor_ok(v, ldv, Hkv, D)) return AGQ_EINVAL;
    if (q && (!tensor_ok(q, ldq, Hq, D) || !tensor_ok(q_out, ldqo, Hq, D))) return AGQ_EINVAL;
    if (k_out && !tensor_ok(k_out, ldko, Hkv, D)) return AGQ_EINVAL;
    const AgqKvAppend a = {cache->k, cache->v, cache->k_exp, cache->v_exp, cache->n_pages, Hkv, D, (int)cache->page, q, k, v, q_out, k_out,
                           ldq, ldk, ldv, ldqo, ldko, T, Hq, P, pos, slot, rope_cos, rope_sin};
    return hip_status(agq_launch_kv_append(a, stream));
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
