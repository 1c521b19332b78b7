// Attention of each request's newest tokens over its pages of the 8-bit cache.
//
// Scores transposed, S^T = K Q^T: a 16 x 16 tile of the matrix instruction holds sixteen keys by sixteen rows (a row: one
// new token and one query head; the heads that share a key head are rows of one tile, so the cache is read once for all of
// them).  A lane then owns one row, and in every chunk of 64 keys the sixteen keys of its lane group, which is just what the
// second product, O^T = V^T P^T, wants from that lane: the probabilities never leave their registers.  Which key a tile's
// row stands for is free, so the keys are dealt out such that a lane's sixteen are neighbours: its bytes of V (kept [D, token]
// in a page) are one load, and so is its piece of a key.  Nothing goes through LDS but the join of the wavefronts.
// A page's scale of K is a factor of the scores.  Its scale of V is added to the exponent: the weight of key j is
// w = 2^(s_j + e_v - M), M the running maximum of s_j + e_v, so the products of pages with different scales add up in one
// accumulator.  w goes into the product as fp16 times 2^15, because the matrix instruction takes both operands in 16 bits: down
// to 2^-29 of the largest weight it has all eleven bits (off by 2^-11 of it at most, and as often up as down); sums, maxima
// and accumulators are fp32.  The softmax's sum is that of w 2^-e_v before w's rounding: on a page of small values w may be
// nothing in fp16, as it is in the product, while w 2^-e_v is most of the sum (exponents lie 40 powers of two apart at most
// where agq_kv_append made them, so w is a normal fp32 number for keys down to 2^-100 of the loudest).
// w's exponent is the score's difference to the lane's largest in the chunk, taken before the scale, and that one's to M: neither is
// above 0 whatever the rounding, so scores of any size (an fp16 query of 60000 makes them up to 2^36) leave weights in fp16's range.
//
// Bound and figures.  Long caches: memory; 4 requests of 60000 to 131072 tokens, 8 key heads of 128, 827 MB in 143 us,
// 5.8 TB/s (a plain read reaches 6.05), and 5 for the join, in a trace; 149 one call after the other, 155 in a replayed graph.
// Many requests of all lengths up to 4096, 64 of them, 100 MB, 26.6 us with the join: a chunk's bytes take 2.7 us to come.
// One request of 1000 tokens, 10.3 us: what 32 CUs can have on
// its way, the launch and the join of the wavefronts.  Bytes requested two chunks ahead change nothing where the registers
// hold them (D = 64) and spill otherwise (13.9 us); so do sixteen wavefronts to a workgroup (23 us) and three workgroups to a
// CU (64 requests, 30.8).
#include "agq_device.h"
#include "agq_internal.h"

#include <type_traits>

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -1e37f;       // the maximum of no keys; scores are above -2^119 with a scale of 2^24 and exponents of 64
constexpr float kUpLog2 = 15.0f;      // weights are 2^15 times what they are, in sums and product alike

struct KvArgs {
    const _Float16 *q;
    _Float16 *o;
    const int32_t *cu_q, *kv_len, *table;
    const int8_t *kc, *vc, *ke, *ve;
    float *part;          // [split][token][query head][D]
    float2 *part_ml;      // [split][token][query head]: maximum, sum
    int64_t ldq, ldo, max_pages;
    float scale;          // log2(e) times the softmax's factor
    float per_piece;      // 1 / pieces
    int T, B, Hq, Hkv, group, page_log2, n_pages, splits, split_keys, row_tiles, pieces;
};

// Eight codes of K as fp16: code + 128 is the low byte of a half, a subnormal, 2^-24 times itself; three instructions for
// four codes.  The factor and 128 times the row's sum of q come out of the score, which is off by the roundings of a sum
// 128 times |q|_1 in size for it, as if every code were that large.
__device__ __forceinline__ half8_t widen_k(uint32_t w0, uint32_t w1) {
    const uint32_t u0 = w0 ^ 0x80808080u, u1 = w1 ^ 0x80808080u;
    const uint4_t h = {__builtin_amdgcn_perm(0u, u0, 0x0c010c00u), __builtin_amdgcn_perm(0u, u0, 0x0c030c02u),
                       __builtin_amdgcn_perm(0u, u1, 0x0c010c00u), __builtin_amdgcn_perm(0u, u1, 0x0c030c02u)};
    return __builtin_bit_cast(half8_t, h);
}
constexpr float kCode = 16777216.0f;  // 2^24
constexpr float kLowest = -0x1p10f;   // below every score in that form: 128 * 255 * 2^16 / 2^24 at most
// Eight codes of V as fp16, exactly: 1024 + (code + 128) - 1152.  (K's form would leave an error of 128 times the rounding
// of the weights' sum in an output whose values are all small.)
__device__ __forceinline__ half8_t widen_v(uint32_t w0, uint32_t w1) {
    const uint32_t u0 = w0 ^ 0x80808080u, u1 = w1 ^ 0x80808080u;
    const uint4_t h = {__builtin_amdgcn_perm(0x64646464u, u0, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, u0, 0x04030402u),
                       __builtin_amdgcn_perm(0x64646464u, u1, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, u1, 0x04030402u)};
    return __builtin_bit_cast(half8_t, h) - (_Float16)1152.0f;
}

// how many workgroups share the keys of a request of L tokens
__device__ __forceinline__ int splits_of(int L, int split_keys, int splits) {
    return min(max((int)(((uint32_t)L + (uint32_t)split_keys - 1) / (uint32_t)split_keys), 1), splits);
}

struct Request {
    int first, n, L;      // its first token in the batch, its new tokens, its tokens in the cache
};
__device__ __forceinline__ Request request_of(const KvArgs &a, int b) {
    const int q0 = min(max(a.cu_q[b], 0), a.T), q1 = min(max(a.cu_q[b + 1], 0), a.T);
    const int64_t cap = a.max_pages << a.page_log2;
    return {q0, q1 - q0, (int)min((int64_t)max(a.kv_len[b], 0), cap)};
}

// Keys of a piece.  pieces != 0: the least number, not below split_keys, with which the requests (64 at most) make no more than
// that many pieces, one for every CU; lengths are known here only.  (4 requests of 60000 to 131072 tokens: with the keys that
// 131072 each would need, a quarter of the CUs has none.)
__device__ __forceinline__ int piece_keys(const KvArgs &a) {
    if (a.pieces == 0) return a.split_keys;
    const int lane = threadIdx.x & 63;
    const int64_t cap = a.max_pages << a.page_log2;
    const int L = lane < a.B ? (int)min((int64_t)max(a.kv_len[lane], 0), cap) : 0;
    const int64_t total = ((int64_t)__builtin_amdgcn_readlane(agq_wave_scan(L >> 8), 63) << 8) + __builtin_amdgcn_readlane(agq_wave_scan(L & 255), 63);
    int keys = max(a.split_keys, (int)((float)total * a.per_piece));
    for (;;) {
        keys = (keys + 255) & ~255;
        const int n = lane < a.B ? splits_of(L, keys, a.splits) : 0;
        if (__builtin_amdgcn_readlane(agq_wave_scan(n), 63) <= a.pieces) return keys;
        keys += keys >> 4;                                                // B <= pieces / 2: ends with a piece for each at the latest
    }
}

// The idx-th piece of all requests' keys, requests one after the other; b = -1: there are fewer.  So the workgroups that find
// none are the last ones: spread over the others they would hold up places on the CUs (64 requests of 16 to 4096 tokens, at most
// eight pieces of 512 keys each: 29 us).
struct Unit {
    int b, split;
};
__device__ __forceinline__ Unit unit_of(const KvArgs &a, int idx, int split_keys) {
    const int lane = threadIdx.x & 63;
    const int64_t cap = a.max_pages << a.page_log2;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + lane;
        const int n = b < a.B ? splits_of((int)min((int64_t)max(a.kv_len[b], 0), cap), split_keys, a.splits) : 0;
        const int up = before + agq_wave_scan(n);
        const unsigned long long over = __ballot(up > idx);
        if (over) {
            const int src = __ffsll((long long)over) - 1;
            return {b0 + src, idx - __builtin_amdgcn_readlane(up - n, src)};
        }
        before = __builtin_amdgcn_readlane(up, 63);
    }
    return {-1, 0};
}

// One workgroup of NW wavefronts (four or eight): NQ tiles of sixteen rows of one key head of one request, over one split of
// its keys; the wavefronts take the chunks of 64 keys in turn.
template <int D, int NQ, int NW>
__global__ __launch_bounds__(NW * 64, 2) void attn_kv_kernel(const KvArgs a) {
    constexpr int KH = D / 64, DT = D / 16, ROWS = 16 * NQ, PAD = D + 4;
    __shared__ __attribute__((aligned(16))) float join[4 * 16 * PAD];
    __shared__ float2 ml[NW * ROWS];                                      // maxima and sums
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int head = blockIdx.x, tile0 = blockIdx.z;
    int b = blockIdx.y, split = 0;
    const int split_keys = piece_keys(a);
    if (a.splits > 1) {
        const Unit u = unit_of(a, blockIdx.y, split_keys);
        if (u.b < 0) return;
        b = u.b, split = u.split;
    }
    // The request's numbers and the first chunks' page numbers are requested together.  Pages: of the keys that the lane loads
    // ((i / 4) * 16 + 4 t + i % 4 for tile t), and of those it owns; what the table says behind the last key does not
    // matter: the mask keeps it out.
    const int32_t *table = a.table + (int64_t)b * a.max_pages;
    const int page1 = (1 << a.page_log2) - 1, k0 = split * split_keys, c0 = (k0 >> 6) + wave;
    auto page_of = [&](int key) { return table[min(key >> a.page_log2, (int)a.max_pages - 1)]; };
    auto inside = [&](int p) { return (unsigned)p < (unsigned)a.n_pages; };
    int first[4] = {page_of(c0 * 64 + (i >> 2) * 16), page_of(c0 * 64 + g * 16), page_of((c0 + NW) * 64 + (i >> 2) * 16), page_of((c0 + NW) * 64 + g * 16)};
    const Request rq = request_of(a, b);
    const int ns = splits_of(rq.L, split_keys, a.splits), rows = rq.n * a.group;

    const half2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
    for (int tile = tile0; tile * ROWS < rows; tile += a.row_tiles) {
        // the rows' queries as the second operand of the first product: lane (row i, group g) holds d = 64 h + 16 g + 0..15
        half8_t q[NQ][KH][2];
        float q128[NQ];            // 128 times the sum of the row
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
            float sum = 0.0f;
#pragma unroll
            for (int h = 0; h < KH; ++h)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) sum = __builtin_amdgcn_fdot2(half2_t{q[n][h][s][e], q[n][h][s][e + 1]}, ones, sum, false);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            q128[n] = 128.0f * sum;
        }
        const int t_first = tile * ROWS / a.group, t_last = min(tile * ROWS + ROWS, rows) - 1;
        const int all_see = rq.L - rq.n + t_first + 1;                    // keys that every row of the tile sees
        const int k1 = min(split == ns - 1 ? rq.L : k0 + split_keys, rq.L - rq.n + t_last / a.group + 1);

        float M[NQ], l[NQ];                                               // maximum, sum of w 2^-e_v
        float4_t o[NQ][DT];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            M[n] = kNone, l[n] = 0.0f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[n][d] = float4_t{};
        }
        // The chunk's bytes: requested a chunk ahead, each as soon as the registers of the one before are free; its page numbers two
        // chunks ahead.  Loads return in the order of their requests: page numbers and scales come before the keys, so that
        // nothing waits for the values but their product.
        uint4 kraw[4][KH], vraw[DT];
        int ek = 0, ev = 0, pk1, pv1;                                       // scales of this chunk; page numbers of the next one
        bool there = true;                                                  // the lane's keys have a page
        auto load_k = [&](int c) {
            const int64_t at = (int64_t)(inside(pv1) ? pv1 : 0) * a.Hkv + head;
            ek = a.ke[at], ev = a.ve[at];
            const int8_t *src = a.kc + ((((int64_t)(inside(pk1) ? pk1 : 0) * a.Hkv + head) << a.page_log2) + ((c * 64 + (i >> 2) * 16) & page1) + (i & 3)) * D + 16 * g;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int h = 0; h < KH; ++h) kraw[t][h] = *reinterpret_cast<const uint4 *>(src + t * 4 * D + h * 64);
        };
        auto load_v = [&](int c) {
            const int8_t *src = a.vc + ((((int64_t)(inside(pv1) ? pv1 : 0) * a.Hkv + head) * D + i) << a.page_log2) + ((c * 64 + g * 16) & page1);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                vraw[d] = *reinterpret_cast<const uint4 *>(src);
                src += 16 << a.page_log2;
                // two tiles of rows: one address instead of eight, for the registers (eleven in memory otherwise; 64 requests of
                // 8 new tokens, lengths 16 to 4096, 41.1 -> 39.9 us; one tile of rows, which has them, is 5 % slower for it)
                if constexpr (NQ == 2) asm volatile("" : "+v"(src));
            }
        };
        auto chunk = [&](int c, auto more_tag) {
            constexpr bool more = decltype(more_tag)::value;
            const int key_v = c * 64 + g * 16;
            int pk2, pv2;
            if constexpr (more) pk2 = page_of((c + 2 * NW) * 64 + (i >> 2) * 16), pv2 = page_of((c + 2 * NW) * 64 + g * 16);

            float4_t s[NQ][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][t] = float4_t{};
#pragma unroll
                for (int h = 0; h < KH; ++h) {
                    const half8_t a0 = widen_k(kraw[t][h].x, kraw[t][h].y), a1 = widen_k(kraw[t][h].z, kraw[t][h].w);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, q[n][h][0], s[n][t], 0, 0, 0);
                        s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, q[n][h][1], s[n][t], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);               // the fp16 form of a tile only lives that long
            }
            const int e_k = min(max(ek, -64), 64), e_v = min(max(ev, -64), 64);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) load_k(c + NW);
            __builtin_amdgcn_sched_barrier(0);
            const float sk = __builtin_amdgcn_ldexpf(a.scale, e_k), sv = (float)e_v, inv = __builtin_amdgcn_ldexpf(1.0f, -e_v);
            const bool masked = c * 64 + 64 > all_see || __any(!there);
            half8_t p[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                if (masked) {
                    asm volatile("");                                     // a branch, not selects in every chunk
                    const int left = there ? seen[n] - key_v : 0;         // of the lane's sixteen keys, those that its row sees
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][t][r] = t * 4 + r < left ? s[n][t][r] : -INFINITY;
                }
                float top = -INFINITY;                                    // the sixteen have one page and so one scale
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, s[n][t][r]);
                const float sk24 = sk * kCode, most = fmaxf(top, kLowest), mine = fmaf(top, sk24, fmaf(-sk, q128[n], sv));
                top = fmaxf(mine, __shfl_xor(mine, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any(top > M[n])) {
                    const float to = fmaxf(M[n], top), f = __builtin_amdgcn_exp2f(M[n] - to);
                    M[n] = to;
                    l[n] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] *= f;
                }
                const float off = mine - M[n] + kUpLog2;                  // of the lane's largest, kUpLog2 at most whatever its size
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const float w0 = __builtin_amdgcn_exp2f(fmaf(s[n][k >> 2][k & 3] - most, sk24, off));
                    const float w1 = __builtin_amdgcn_exp2f(fmaf(s[n][k >> 2][(k & 3) + 1] - most, sk24, off));
                    sum += w0 + w1;
                    p[n][k >> 3][k & 7] = (_Float16)w0;
                    p[n][k >> 3][(k & 7) + 1] = (_Float16)w1;
                }
                l[n] = fmaf(sum, inv, l[n]);
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const half8_t a0 = widen_v(vraw[d].x, vraw[d].y), a1 = widen_v(vraw[d].z, vraw[d].w);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0, p[n][0], o[n][d], 0, 0, 0);
                    o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1, p[n][1], o[n][d], 0, 0, 0);
                }
                if (d % 2) __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) {
                load_v(c + NW);
                there = inside(pv1);
                pk1 = pk2, pv1 = pv2;
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        int c = c0;
        if (c * 64 < k1) {
            pk1 = first[0], pv1 = first[1];
            __builtin_amdgcn_sched_barrier(0);
            load_k(c);
            load_v(c);
            there = inside(pv1);
            pk1 = first[2], pv1 = first[3];
            for (; (c + NW) * 64 < k1; c += NW) chunk(c, std::true_type{});
            chunk(c, std::false_type{});
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
            for (int d = 0; d < DT; ++d) o[n][d] *= f;
            float4_t *mine = reinterpret_cast<float4_t *>(join + ((wave & 3) * 16 + i) * PAD + g * 4);
            if constexpr (NW == 8) {                                      // the upper four into the lower four
                if (wave >= 4)
#pragma unroll
                    for (int d = 0; d < DT; ++d) mine[d * 4] = o[n][d];
                __syncthreads();
                if (wave < 4)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] += mine[d * 4];
            }
            if (wave < 4)
#pragma unroll
                for (int d = 0; d < DT; ++d) mine[d * 4] = o[n][d];
            __syncthreads();
            int it = threadIdx.x;
            asm volatile("" : "+v"(it));                                  // addresses of the stores: made here, no registers before
            for (; it < 16 * (D / 4); it += NW * 64) {
                const int rr = it / (D / 4), d = it % (D / 4) * 4, r = tile * ROWS + n * 16 + rr;
                if (r >= rows) continue;
                float top = kNone, sum = 0.0f;
                for (int w = 0; w < NW; ++w) top = fmaxf(top, ml[w * ROWS + n * 16 + rr].x);
                for (int w = 0; w < NW; ++w) {
                    const float2 m = ml[w * ROWS + n * 16 + rr];
                    sum += m.y * __builtin_amdgcn_exp2f(m.x - top);
                }
                float4_t acc = {};
                for (int w = 0; w < 4; ++w) acc += *reinterpret_cast<const float4_t *>(join + (w * 16 + rr) * PAD + d);
                const int t = rq.first + r / a.group, h = head * a.group + r % a.group;
                if (ns == 1) {
                    const float f1 = sum == 0.0f ? 0.0f : 1.0f / sum;
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
    const int ns = splits_of(rq.L, piece_keys(a), a.splits), lane = threadIdx.x & 63;
    if (ns == 1) return;
    constexpr int W = D / 64, AHEAD = 8;
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rq.n * a.Hq; r += gridDim.x * 4) {
        const int64_t row0 = (int64_t)rq.first * a.Hq + r, step = (int64_t)a.T * a.Hq;
        // the splits' maxima and sums, one lane each (in rounds of 64), then their outputs, eight loads at a time
        float top = kNone, sum = 0.0f, acc[W] = {};
        for (int s0 = 0; s0 < ns; s0 += 64) {
            const bool on = s0 + lane < ns;
            const float2 ml = on ? a.part_ml[row0 + (s0 + lane) * step] : make_float2(kNone, 0.0f);
            float most = ml.x;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
            const float to = fmaxf(top, most), f0 = __builtin_amdgcn_exp2f(top - to), f = on ? __builtin_amdgcn_exp2f(ml.x - to) : 0.0f;
            float part = ml.y * f;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) part += __shfl_xor(part, m);
            sum = sum * f0 + part;
            top = to;
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] *= f0;
            const int here = min(ns - s0, 64);
            for (int s = 0; s < here; s += AHEAD) {
                float x[AHEAD][W], w[AHEAD];
#pragma unroll
                for (int e = 0; e < AHEAD; ++e) {
                    const float *src = a.part + (row0 + (s0 + min(s + e, here - 1)) * step) * D + lane * W;
#pragma unroll
                    for (int j = 0; j < W; ++j) x[e][j] = src[j];
                    w[e] = s + e < here ? __shfl(f, min(s + e, 63)) : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < AHEAD; ++e)
#pragma unroll
                    for (int j = 0; j < W; ++j) acc[j] = fmaf(x[e][j], w[e], acc[j]);
            }
        }
        const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int t = rq.first + r / a.Hq, h = r % a.Hq;
        _Float16 y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) y[j] = (_Float16)(acc[j] * f);
        _Float16 *dst = a.o + (int64_t)t * a.ldo + h * D + lane * W;
        if constexpr (W == 2) *reinterpret_cast<uint32_t *>(dst) = __builtin_bit_cast(uint32_t, y);
        else *dst = y[0];
    }
}

template <int D, int NQ, int NW>
int launch(const KvArgs &a, hipStream_t st) {
    attn_kv_kernel<D, NQ, NW><<<dim3((unsigned)a.Hkv, (unsigned)(a.pieces ? a.pieces : a.B * a.splits), (unsigned)a.row_tiles), NW * 64, 0, st>>>(a);
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
    a.splits = sp.splits, a.split_keys = sp.split_keys, a.row_tiles = sp.row_tiles, a.pieces = sp.pieces, a.per_piece = sp.pieces ? 1.0f / (float)sp.pieces : 0.0f;
    a.part = (float *)workspace;
    a.part_ml = (float2 *)(a.part + (size_t)a.splits * p.T * p.Hq * p.D);
    hipStream_t st = (hipStream_t)stream;
    int err;
    if (p.D == 128)
        err = sp.tiles == 2 ? sp.waves == 8 ? launch<128, 2, 8>(a, st) : launch<128, 2, 4>(a, st) : sp.waves == 8 ? launch<128, 1, 8>(a, st) : launch<128, 1, 4>(a, st);
    else
        err = sp.tiles == 2 ? sp.waves == 8 ? launch<64, 2, 8>(a, st) : launch<64, 2, 4>(a, st) : sp.waves == 8 ? launch<64, 1, 8>(a, st) : launch<64, 1, 4>(a, st);
    if (err || a.splits == 1) return err;
    const int64_t rows = (p.max_q > 0 ? p.max_q : 1) * p.Hq;
    const dim3 grid((unsigned)(rows < 4 * 1024 ? (rows + 3) / 4 : 1024), (unsigned)p.B);
    if (p.D == 128)
        attn_kv_join_kernel<128><<<grid, 256, 0, st>>>(a);
    else
        attn_kv_join_kernel<64><<<grid, 256, 0, st>>>(a);
    return (int)hipGetLastError();
}
