// Attention over whole prompts, packed one behind the other, causal or not, with grouped heads.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four wavefronts takes 128 queries
// of one head, a wavefront 32 of them; the keys and values pass through LDS, 64 at a time.  Scores transposed: S^T = K Q^T
// on 32 x 32 x 16 matrix instructions leaves a lane with one query's scores of sixteen keys out of 32, and O^T = V^T P^T
// takes the probabilities from those very registers, if the keys of its operand V^T are dealt out in the same order; that
// operand comes out of LDS by transposing reads.  Sums, maxima and accumulators are fp32; probabilities go into the second
// product as fp16 times 2^10 (off by 2^-11 of it at most, down to 2^-24 of the largest).
#include "agq_device.h"
#include "agq_internal.h"

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -1e30f;      // the maximum of no keys
constexpr float kUp = 1024.0f;       // 2^10: probabilities in the second product
constexpr int kRows = 128, kKeys = 64;

struct PackedArgs {
    const _Float16 *q, *k, *v;
    _Float16 *o;
    const int32_t *cu_q, *cu_k;
    int64_t ldq, ldk, ldv, ldo;
    float scale;                     // log2(e) times the softmax's factor
    int Tq, Tk, B, Hq, group, causal;
};

struct Tile {
    int b, q0, n, m, k0, row;        // sequence, its first query and their number, its keys and the first of them, the tile's first row
};
// The idx-th tile of `rows` queries, sequences one after the other, a sequence's last tile (the longest under a causal mask)
// first; b = -1: there are fewer.  Offsets are taken into the tensors' bounds.
__device__ __forceinline__ Tile tile_of(const PackedArgs &a, int idx, int rows) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + lane;
        int q0 = 0, n = 0;
        if (b < a.B) {
            q0 = min(max(a.cu_q[b], 0), a.Tq);
            n = max(min(max(a.cu_q[b + 1], 0), a.Tq) - q0, 0);
        }
        const int tiles = (n + rows - 1) / rows;
        int up = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(up, d);
            up += lane >= d ? u : 0;
        }
        const unsigned long long over = __ballot(before + up > idx);
        if (over) {
            const int src = __ffsll((long long)over) - 1;
            Tile t;
            t.b = b0 + src;
            t.q0 = __shfl(q0, src);
            t.n = __shfl(n, src);
            const int last = __shfl(before + up, src) - 1;       // the sequence's last tile is its number 0
            t.row = (last - idx) * rows;
            t.k0 = min(max(a.cu_k[t.b], 0), a.Tk);
            t.m = max(min(max(a.cu_k[t.b + 1], 0), a.Tk) - t.k0, 0);
            return t;
        }
        before += __shfl(up, 63);
    }
    Tile t = {};
    t.b = -1;
    return t;
}

// four keys of one column of a [key][d] tile in LDS: lanes 4 r + c of a group of sixteen name row r's columns 4 c .. 4 c + 3,
// lane j receives column j of the four rows
__device__ __forceinline__ short4_t read_tr(const _Float16 *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)p);
}

template <int D>
__global__ __launch_bounds__(256) void attn_packed_kernel(const PackedArgs a) {
    constexpr int KS = D / 16, DT = D / 32, CH = D / 8;            // steps of the first product, row tiles of the second, 16-byte pieces of a row
    constexpr int LOADS = kKeys * CH / 256;
    __shared__ __attribute__((aligned(16))) _Float16 ks[kKeys * D], vs[kKeys * D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 31, h = lane >> 5;
    const int head = blockIdx.x % a.Hq, kv = head / a.group;
    const Tile tl = tile_of(a, blockIdx.x / a.Hq, kRows);
    if (tl.b < 0) return;
    const int row = tl.row + wave * 32 + i;                        // the lane's query
    const bool on = row < tl.n;
    half8_t q[KS];
    {
        const _Float16 *src = a.q + (int64_t)(tl.q0 + (on ? row : 0)) * a.ldq + head * D + 8 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = *reinterpret_cast<const half8_t *>(src + 16 * s);
            if (!on) q[s] = half8_t{};
        }
    }
    const int past = tl.m - tl.n;                                  // query r sees keys up to past + r
    const int seen = a.causal ? min(past + row + 1, tl.m) : tl.m;
    const int rows_here = min(tl.n - tl.row, kRows);
    const int all_keys = a.causal ? min(past + tl.row + rows_here, tl.m) : tl.m;              // keys that some row of the workgroup sees
    const int wave_keys = a.causal ? min(past + tl.row + wave * 32 + 32, tl.m) : tl.m;        // ... of the wavefront
    const int wave_all = a.causal ? past + tl.row + wave * 32 + 1 : tl.m;                     // keys that every row of it sees
    const _Float16 *kbase = a.k + (int64_t)tl.k0 * a.ldk + kv * D, *vbase = a.v + (int64_t)tl.k0 * a.ldv + kv * D;

    float M = kNone, l = 0.0f;
    float16_t o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = float16_t{};

    uint4 kr[LOADS], vr[LOADS];
    auto load = [&](int key0) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int it = j * 256 + tid, r = key0 + it / CH, c = it % CH;
            // rows behind the sequence are not read: another sequence's, or nobody's
            kr[j] = vr[j] = make_uint4(0u, 0u, 0u, 0u);
            if (r < tl.m) {
                kr[j] = *reinterpret_cast<const uint4 *>(kbase + (int64_t)r * a.ldk + c * 8);
                vr[j] = *reinterpret_cast<const uint4 *>(vbase + (int64_t)r * a.ldv + c * 8);
            }
        }
    };
    if (all_keys > 0) load(0);
    for (int key0 = 0; key0 < all_keys; key0 += kKeys) {
        __syncthreads();
        bool odd = false;                       // an infinity or NaN among the thread's values
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int it = j * 256 + tid, r = it / CH, c = it % CH;
            *reinterpret_cast<uint4 *>(ks + r * D + ((c ^ (r & 7)) * 8)) = kr[j];
            *reinterpret_cast<uint4 *>(vs + r * D + ((c ^ ((r & 3) * (D == 128 ? 4 : 2))) * 8)) = vr[j];
            const uint32_t w[4] = {vr[j].x, vr[j].y, vr[j].z, vr[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= (w[e] & 0x7C00u) == 0x7C00u || (w[e] & 0x7C000000u) == 0x7C000000u;
        }
        // Such values under the mask must not reach the rows that do not see them (0 times an infinity is NaN); they go in by
        // the slow way below, and only in tiles that the mask cuts
        const bool slow = __syncthreads_or(odd) && key0 + kKeys > (a.causal ? past + tl.row + 1 : tl.m);
        if (key0 + kKeys < all_keys) load(key0 + kKeys);
        if (key0 >= wave_keys) continue;

        float16_t s[2] = {};
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const int r = half * 32 + i;
                const half8_t kf = *reinterpret_cast<const half8_t *>(ks + r * D + (((st * 2 + h) ^ (r & 7)) * 8));
                s[half] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, q[st], s[half], 0, 0, 0);
            }
        const bool masked = key0 + kKeys > wave_all;
        float top = kNone;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = s[half][r] * a.scale;
                const int key = key0 + half * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                if (masked) x = key < seen ? x : -INFINITY;
                s[half][r] = x;
                top = fmaxf(top, x);
            }
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > M)) {
            const float to = fmaxf(M, top), f = __builtin_amdgcn_exp2f(M - to);
            M = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= f;
        }
        half8_t p[4];
        float sum = 0.0f;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = __builtin_amdgcn_exp2f(s[half][r] - M);
                sum += w;
                p[half * 2 + (r >> 3)][r & 7] = (_Float16)(w * kUp);
            }
        l += sum;
        // O^T += V^T P^T; the lane's keys of step st: 16 st + 8 (e / 4) + 4 h + e % 4
        const int tr_row = 4 * h + ((lane & 15) >> 2), tr_col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                short4_t part[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = st * 16 + e * 8 + tr_row, col = d * 32 + tr_col;
                    part[e] = read_tr(vs + r * D + (((col >> 3) ^ ((r & 3) * (D == 128 ? 4 : 2))) * 8) + (col & 7));
                }
                short vfr[8] = {part[0].x, part[0].y, part[0].z, part[0].w, part[1].x, part[1].y, part[1].z, part[1].w};
                half8_t vf = __builtin_bit_cast(half8_t, vfr);
                if (slow) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) vf[e] = (((uint16_t)vfr[e]) & 0x7C00u) == 0x7C00u ? (_Float16)0.0f : vf[e];
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p[st], o[d], 0, 0, 0);
            }
        if (slow) {
            for (int r = 0; r < kKeys && key0 + r < seen; ++r)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int col = d * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
                        const _Float16 x = vs[r * D + (((col >> 3) ^ ((r & 3) * (D == 128 ? 4 : 2))) * 8) + (col & 7)];
                        if ((__builtin_bit_cast(uint16_t, x) & 0x7C00u) == 0x7C00u) o[d][e] += (float)x;
                    }
        }
    }
    l += __shfl_xor(l, 32);
    if (!on) return;
    const float f = l == 0.0f ? 0.0f : 1.0f / (l * kUp);
    _Float16 *dst = a.o + (int64_t)(tl.q0 + row) * a.ldo + head * D + 4 * h;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = (_Float16)(o[d][e * 4 + j] * f);
            *reinterpret_cast<uint2 *>(dst + d * 32 + e * 8) = __builtin_bit_cast(uint2, y);
        }
}

}  // namespace

int agq_launch_attn_packed(const AgqAttnPacked &p, void *stream) {
    PackedArgs a;
    a.q = (const _Float16 *)p.q, a.k = (const _Float16 *)p.k, a.v = (const _Float16 *)p.v, a.o = (_Float16 *)p.o;
    a.cu_q = p.cu_q, a.cu_k = p.cu_k;
    a.ldq = p.ldq, a.ldk = p.ldk, a.ldv = p.ldv, a.ldo = p.ldo;
    a.scale = p.scale * 1.44269504088896340736f;
    a.Tq = (int)p.Tq, a.Tk = (int)p.Tk, a.B = (int)p.B, a.Hq = (int)p.Hq, a.group = (int)(p.Hq / p.Hkv), a.causal = p.causal;
    const int64_t tiles = p.Tq / kRows + p.B;                       // sum of ceil(n / 128) is not more
    const dim3 grid((unsigned)(tiles * p.Hq));
    if (p.D == 128)
        attn_packed_kernel<128><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else
        attn_packed_kernel<64><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}
