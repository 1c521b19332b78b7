// Attention of each request's newest tokens over its pages of the 8-bit cache.
//
// Scores transposed, S^T = K Q^T: a 16 x 16 tile of the matrix instruction holds sixteen keys by sixteen rows (a row: one
// new token and one query head; the heads that share a key head are rows of one tile, so the cache is read once for all of
// them).  A lane then owns one row, and in every chunk of 64 keys the sixteen keys of its lane group, which is just what the
// second product, O^T = V^T P^T, wants from that lane: the probabilities never leave their registers.  Which key a tile's
// row stands for is free, so the keys are dealt out such that a lane's sixteen are neighbours: its bytes of V (kept [D, token]
// in a page) are one load, and so is its piece of a key.  Nothing goes through LDS but the join of the wavefronts.
// Codes become fp16 exactly (1024 + code + 128 - 1152); a page's scale of K is a factor of the scores.  Its scale of V is
// added to the exponent: the weight of key j is w = 2^(s_j + e_v - M), M the running maximum of s_j + e_v, so the products of
// pages with different scales add up in one accumulator, and the softmax's sum is that of w 2^-e_v.  w goes into the product
// as fp16 times 2^15: down to 2^-29 of the largest weight it has all eleven bits (off by 2^-11 of it at most, and as often up
// as down); sums, maxima and accumulators are fp32.
#include "agq_device.h"
#include "agq_internal.h"

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -1e30f;       // the maximum of no keys
constexpr float kUp = 32768.0f;       // 2^15: weights in the second product

struct KvArgs {
    const _Float16 *q;
    _Float16 *o;
    const int32_t *cu_q, *kv_len, *table;
    const int8_t *kc, *vc, *ke, *ve;
    float *part;          // [split][token][query head][D]
    float2 *part_ml;      // [split][token][query head]: maximum, sum
    int64_t ldq, ldo, max_pages;
    float scale;          // log2(e) times the softmax's factor
    int T, B, Hq, Hkv, group, page_log2, n_pages, splits, split_keys, row_tiles;
};

// four codes -> four fp16
__device__ __forceinline__ void widen4(uint32_t w, half2_t &a, half2_t &b) {
    const uint32_t u = w ^ 0x80808080u;
    const half2_t off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
    b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
}
__device__ __forceinline__ half8_t widen8(uint32_t w0, uint32_t w1) {
    half2_t a, b, c, d;
    widen4(w0, a, b);
    widen4(w1, c, d);
    return half8_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// how many workgroups share the keys of a request of L tokens
__device__ __forceinline__ int splits_of(int L, int split_keys, int splits) {
    return min(max((L + split_keys - 1) / split_keys, 1), splits);
}

struct Request {
    int first, n, L;      // its first token in the batch, its new tokens, its tokens in the cache
};
__device__ __forceinline__ Request request_of(const KvArgs &a, int b) {
    const int q0 = min(max(a.cu_q[b], 0), a.T), q1 = min(max(a.cu_q[b + 1], 0), a.T);
    const int64_t cap = a.max_pages << a.page_log2;
    return {q0, q1 - q0, (int)min((int64_t)max(a.kv_len[b], 0), cap)};
}

// One workgroup of NW wavefronts: NQ tiles of sixteen rows of one key head of one request, over one split of its keys;
// the wavefronts take the chunks of 64 keys in turn.
template <int D, int NQ, int NW>
__global__ __launch_bounds__(NW * 64) void attn_kv_kernel(const KvArgs a) {
    constexpr int KH = D / 64, DT = D / 16, ROWS = 16 * NQ;
    __shared__ __attribute__((aligned(16))) float join[NW * 16 * D];
    __shared__ float2 ml[NW * ROWS];                                      // maxima and sums
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    unsigned id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile0 = id % a.row_tiles;
    id /= a.row_tiles;
    const int head = id % a.Hkv, b = id / a.Hkv;
    const Request rq = request_of(a, b);
    const int ns = splits_of(rq.L, a.split_keys, a.splits), rows = rq.n * a.group;
    if (split >= ns) return;
    const int32_t *table = a.table + (int64_t)b * a.max_pages;

    for (int tile = tile0; tile * ROWS < rows; tile += a.row_tiles) {
        // the rows' queries as the second operand of the first product: lane (row i, group g) holds d = 64 h + 16 g + 0..15
        half8_t q[NQ][KH][2];
        int seen[NQ];              // keys that the lane's row sees
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int r = tile * ROWS + n * 16 + i, t = r / a.group, hh = r - t * a.group;
            const bool on = r < rows;
            seen[n] = on ? rq.L - rq.n + t + 1 : 0;
            const _Float16 *src = a.q + (int64_t)(rq.first + (on ? t : 0)) * a.ldq + (head * a.group + (on ? hh : 0)) * D + 16 * g;
#pragma unroll
            for (int h = 0; h < KH; ++h)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    q[n][h][s] = *reinterpret_cast<const half8_t *>(src + 64 * h + 8 * s);
                    if (!on) q[n][h][s] = half8_t{};
                }
        }
        const int t_first = tile * ROWS / a.group, t_last = min(tile * ROWS + ROWS, rows) - 1;
        const int all_see = rq.L - rq.n + t_first + 1;                    // keys that every row of the tile sees
        const int k0 = split * a.split_keys;
        const int k1 = min(split == ns - 1 ? rq.L : k0 + a.split_keys, rq.L - rq.n + t_last / a.group + 1);

        float M[NQ], l[NQ];
        float4_t o[NQ][DT];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            M[n] = kNone, l[n] = 0.0f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[n][d] = float4_t{};
        }
        for (int c = (k0 >> 6) + wave; c * 64 < k1; c += NW) {
            // pages: of the keys that the lane loads ((i / 4) * 16 + 4 t + i % 4 for tile t), and of those that it owns
            auto page_of = [&](int key) {
                const int at = key >> a.page_log2;
                const int p = key < rq.L ? table[at] : -1;
                return (unsigned)p < (unsigned)a.n_pages ? p : -1;
            };
            const int page1 = (1 << a.page_log2) - 1;
            const int key_k = c * 64 + (i >> 2) * 16, key_v = c * 64 + g * 16;
            const int pk = page_of(key_k), pv = page_of(key_v);
            const int8_t *kp = a.kc + ((((int64_t)max(pk, 0) * a.Hkv + head) << a.page_log2) + (key_k & page1) + (i & 3)) * D + 16 * g;
            const int8_t *vp = a.vc + (((int64_t)max(pv, 0) * a.Hkv + head) << a.page_log2) * D + (key_v & page1);
            uint4 kraw[4][KH], vraw[DT];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int h = 0; h < KH; ++h) kraw[t][h] = *reinterpret_cast<const uint4 *>(kp + t * 4 * D + h * 64);
#pragma unroll
            for (int d = 0; d < DT; ++d) vraw[d] = *reinterpret_cast<const uint4 *>(vp + ((int64_t)(d * 16 + i) << a.page_log2));
            const int64_t e_at = (int64_t)max(pv, 0) * a.Hkv + head;
            const int ek = min(max((int)a.ke[e_at], -64), 64), ev = min(max((int)a.ve[e_at], -64), 64);

            float4_t s[NQ][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][t] = float4_t{};
#pragma unroll
                for (int h = 0; h < KH; ++h) {
                    const half8_t a0 = widen8(kraw[t][h].x, kraw[t][h].y), a1 = widen8(kraw[t][h].z, kraw[t][h].w);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, q[n][h][0], s[n][t], 0, 0, 0);
                        s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, q[n][h][1], s[n][t], 0, 0, 0);
                    }
                }
            }
            const float sk = __builtin_amdgcn_ldexpf(a.scale, ek), sv = (float)ev, inv = __builtin_amdgcn_ldexpf(1.0f, -ev);
            const bool masked = c * 64 + 64 > all_see || __any(pv < 0);
            half8_t p[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float x[16], top = kNone;
                const int left = pv < 0 ? 0 : seen[n] - key_v;            // of the lane's sixteen keys, those that its row sees
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float y = fmaf(s[n][t][r], sk, sv);
                        if (masked) y = t * 4 + r < left ? y : -INFINITY;
                        x[t * 4 + r] = y;
                        top = fmaxf(top, y);
                    }
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any(top > M[n])) {
                    const float to = fmaxf(M[n], top), f = __builtin_amdgcn_exp2f(M[n] - to);
                    M[n] = to;
                    l[n] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] *= f;
                }
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float w = __builtin_amdgcn_exp2f(x[k] - M[n]);
                    sum += w;
                    p[n][k >> 3][k & 7] = (_Float16)(w * kUp);
                }
                l[n] = fmaf(sum, inv, l[n]);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const half8_t a0 = widen8(vraw[d].x, vraw[d].y), a1 = widen8(vraw[d].z, vraw[d].w);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, p[n][0], o[n][d], 0, 0, 0);
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, p[n][1], o[n][d], 0, 0, 0);
                }
            }
        }
        // the lane groups' sums, then the wavefronts
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (g == 0) ml[wave * ROWS + n * 16 + i] = make_float2(M[n], l[n]);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float most = kNone;
            for (int w = 0; w < NW; ++w) most = fmaxf(most, ml[w * ROWS + n * 16 + i].x);
            const float f = __builtin_amdgcn_exp2f(M[n] - most);
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<float4_t *>(join + (wave * 16 + i) * D + d * 16 + g * 4) = o[n][d] * f;
            __syncthreads();
            for (int it = threadIdx.x; it < 16 * (D / 4); it += NW * 64) {
                const int rr = it / (D / 4), d = it % (D / 4) * 4, r = tile * ROWS + n * 16 + rr;
                if (r >= rows) continue;
                float top = kNone, sum = 0.0f;
                for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[w * ROWS + n * 16 + rr].x);
                float4_t acc = {};
                for (int w = 0; w < NW; ++w) {
                    const float2 m = ml[w * ROWS + n * 16 + rr];
                    sum += m.y * __builtin_amdgcn_exp2f(m.x - top);
                    acc += *reinterpret_cast<const float4_t *>(join + (w * 16 + rr) * D + d);
                }
                const int t = rq.first + r / a.group, h = head * a.group + r % a.group;
                if (ns == 1) {
                    const float f1 = sum == 0.0f ? 0.0f : 1.0f / (sum * kUp);
                    _Float16 y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = (_Float16)(acc[j] * f1);
                    *reinterpret_cast<uint2 *>(a.o + (int64_t)t * a.ldo + h * D + d) = __builtin_bit_cast(uint2, y);
                } else {
                    const int64_t row = ((int64_t)split * a.T + t) * a.Hq + h;
                    *reinterpret_cast<float4_t *>(a.part + row * D + d) = acc;
                    if (d == 0) a.part_ml[row] = make_float2(top, sum);
                }
            }
            __syncthreads();
        }
    }
}

// The splits of a row joined: a wavefront per row (grid: rows of four, requests).
template <int D>
__global__ __launch_bounds__(256) void attn_kv_join_kernel(const KvArgs a) {
    const Request rq = request_of(a, blockIdx.y);
    const int ns = splits_of(rq.L, a.split_keys, a.splits), lane = threadIdx.x & 63;
    if (ns == 1) return;
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rq.n * a.Hq; r += gridDim.x * 4) {
        const int64_t row0 = (int64_t)rq.first * a.Hq + r, step = (int64_t)a.T * a.Hq;
        float top = kNone;
        for (int s = 0; s < ns; ++s) top = fmaxf(top, a.part_ml[row0 + s * step].x);
        float sum = 0.0f, acc[D / 64] = {};
        for (int s = 0; s < ns; ++s) {
            const float2 ml = a.part_ml[row0 + s * step];
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            sum += ml.y * f;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) acc[j] += a.part[(row0 + s * step) * D + lane * (D / 64) + j] * f;
        }
        const float f = sum == 0.0f ? 0.0f : 1.0f / (sum * kUp);
        const int t = rq.first + r / a.Hq, h = r % a.Hq;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) a.o[(int64_t)t * a.ldo + h * D + lane * (D / 64) + j] = (_Float16)(acc[j] * f);
    }
}

template <int D, int NQ, int NW>
int launch(const KvArgs &a, hipStream_t st) {
    attn_kv_kernel<D, NQ, NW><<<dim3((unsigned)((int64_t)a.B * a.Hkv * a.row_tiles * a.splits)), NW * 64, 0, st>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

int agq_launch_attn_kv(const AgqAttnKv &p, const AgqKvSplit &sp, void *workspace, void *stream) {
    KvArgs a;
    a.q = (const _Float16 *)p.q, a.o = (_Float16 *)p.o, a.ldq = p.ldq, a.ldo = p.ldo;
    a.cu_q = p.cu_q, a.kv_len = p.kv_len, a.table = p.block_table, a.max_pages = p.max_pages;
    a.kc = p.k_cache, a.vc = p.v_cache, a.ke = p.k_exp, a.ve = p.v_exp;
    a.scale = p.scale * 1.44269504088896340736f;
    a.T = (int)p.T, a.B = (int)p.B, a.Hq = (int)p.Hq, a.Hkv = (int)p.Hkv, a.group = (int)(p.Hq / p.Hkv);
    a.page_log2 = __builtin_ctz((unsigned)p.page), a.n_pages = (int)p.n_pages;
    a.splits = sp.splits, a.split_keys = sp.split_keys, a.row_tiles = sp.row_tiles;
    a.part = (float *)workspace;
    a.part_ml = (float2 *)(a.part + (size_t)a.splits * p.T * p.Hq * p.D);
    hipStream_t st = (hipStream_t)stream;
    int err;
    if (p.D == 128)
        err = sp.tiles == 1 ? launch<128, 1, 4>(a, st) : launch<128, 2, 4>(a, st);
    else
        err = sp.tiles == 1 ? launch<64, 1, 4>(a, st) : launch<64, 2, 4>(a, st);
    if (err || a.splits == 1) return err;
    const int64_t rows = p.max_q * p.Hq;
    const dim3 grid((unsigned)(rows < 4 * 1024 ? (rows + 3) / 4 : 1024), (unsigned)p.B);
    if (p.D == 128)
        attn_kv_join_kernel<128><<<grid, 256, 0, st>>>(a);
    else
        attn_kv_join_kernel<64><<<grid, 256, 0, st>>>(a);
    return (int)hipGetLastError();
}
