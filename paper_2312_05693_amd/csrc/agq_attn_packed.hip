// Attention over whole prompts, packed one behind the other, causal or not, with grouped heads.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four wavefronts takes 128 queries
// of one head, a wavefront 32 of them; keys and values pass through LDS in sub-tiles of 32.  Scores transposed: S^T = K Q^T
// on 32 x 32 x 16 matrix instructions leaves a lane with one query's scores of sixteen keys out of 32, and O^T = V^T P^T
// takes the probabilities from those very registers, if the keys of its operand V^T are dealt out in the same order; that
// operand comes out of LDS by transposing reads.  Sums, maxima and accumulators are fp32; probabilities go into the second
// product as fp16 times 2^10 (off by 2^-11 of it at most, down to 2^-24 of the largest), because the matrix instruction takes
// both operands in 16 bits.
//
// Bound and figures.  Long prompts: a step of 32 keys has 2 D / 16 matrix instructions of 32 cycles and about as many cycles of
// vector arithmetic, and the two units mostly take turns: 16000 tokens in seven prompts of up to 8191, 32 heads on 8, D = 128,
// 770 to 835 us from card to card, 890 to 970 TFLOP/s (a library product of two matrices of that size class reaches 1264),
// matrix cores busy 54 % of the cycles and the vector ALU 48 %; D = 64, with half the products for the same exponentials, 451
// to 480 us, 780 to 830.  One prompt of 2048 in 40 heads, 59 to 62 us: its longest tiles, 64 steps, take 42 with a CU to
// themselves and 54 in pairs.  A handful of short prompts 7.6 us, of which an empty launch is 1.6.
#include "agq_device.h"
#include "agq_internal.h"

#include <type_traits>

namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint2_t __attribute__((ext_vector_type(2)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr float kNone = -1e30f;      // the maximum of no keys
constexpr float kUpLog2 = 10.0f;     // probabilities are 2^10 times what they are, in sum and product alike
constexpr float kSlack = 5.0f;       // how far a score may lie above the row's reference, in powers of two
constexpr int kRows = 128;

struct PackedArgs {
    const _Float16 *q, *k, *v;
    _Float16 *o;
    const int32_t *cu_q, *cu_k;
    int64_t ldq, ldk, ldv, ldo;
    float *part;                     // [split][token][query head][D]: outputs before the division
    float2 *part_ml;                 // [split][token][query head]: reference and sum
    float scale;                     // log2(e) times the softmax's factor
    int Tq, Tk, B, Hq, group, causal, splits, split_steps;
    int turned;                      // workgroups 256 to here are taken in the opposite order (see launch)
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
        const int up = agq_wave_scan(tiles);
        const unsigned long long over = __ballot(before + up > idx);
        if (over) {
            const int src = __ffsll((long long)over) - 1;
            Tile t;
            t.b = __builtin_amdgcn_readfirstlane(b0 + src);
            t.q0 = __builtin_amdgcn_readlane(q0, src);
            t.n = __builtin_amdgcn_readlane(n, src);
            const int last = __builtin_amdgcn_readlane(before + up, src) - 1;       // the sequence's last tile is its number 0
            t.row = (last - idx) * rows;
            t.k0 = min(max(a.cu_k[t.b], 0), a.Tk);
            t.m = max(min(max(a.cu_k[t.b + 1], 0), a.Tk) - t.k0, 0);
            return t;
        }
        before += __builtin_amdgcn_readlane(up, 63);
    }
    Tile t = {};
    t.b = -1;
    return t;
}

// sub-tiles of 32 keys that some row of the tile sees, and the workgroups that share them
__device__ __forceinline__ int steps_of(const PackedArgs &a, const Tile &t) {
    const int last = min(t.row + kRows, t.n) - 1;
    return (max(a.causal ? min(t.m - t.n + last + 1, t.m) : t.m, 0) + 31) >> 5;
}
__device__ __forceinline__ int splits_of(const PackedArgs &a, const Tile &t) {
    return a.splits == 1 ? 1 : min(max((steps_of(a, t) + a.split_steps - 1) / a.split_steps, 1), a.splits);
}

// what a row's sum is divided by: a row without a key is 0; one that sees keys, but none with a score above -infinity, has no
// softmax and is NaN
__device__ __forceinline__ float inverse_of(float sum, bool sees) {
    return sum == 0.0f ? sees ? __builtin_nanf("") : 0.0f : 1.0f / sum;
}

// four keys of one column of a [key][d] tile in LDS: lanes 4 r + c of a group of sixteen name row r's columns 4 c .. 4 c + 3,
// lane j receives column j of the four rows
__device__ __forceinline__ short4_t read_tr(uint32_t at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)(uintptr_t)at);
}
__device__ __forceinline__ half8_t read_lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) half8_t *)(uintptr_t)at;
}

template <int N>
struct Int {
    static constexpr int value = N;
};
template <int N, int I = 0, class F>
__device__ __forceinline__ void unroll(F &&f) {
    if constexpr (I < N) {
        f(Int<I>{});
        unroll<N, I + 1>(f);
    }
}

// At most VM of this wavefront's copies may still fly (they return in order), its LDS reads are done; then meet the others.
template <int VM>
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | 0x70);   // vmcnt(VM) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Keys go by in sub-tiles of 32.  In step u the scores of sub-tile u + 1 and the product with the values of sub-tile u - 1 run on
// the matrix cores while the vector ALU turns the scores of sub-tile u into probabilities: three independent pieces of
// work, dealt out one matrix instruction at a time.  The wavefronts meet every two steps; copies into LDS run two ahead (rings
// of four).
// Rows' reference: a probability is 2^(c s - off); off is raised to the row's maximum (less 10) only when a score is five
// above it, so the accumulators are seldom rescaled and a weight stays below 2^15.
template <int D>
__global__ __launch_bounds__(256, 2) void attn_packed_kernel(const PackedArgs a) {
    constexpr int KS = D / 16, DT = D / 32;                        // matrix instructions for a sub-tile's scores; d tiles of the output
    constexpr int PIECES = D / 8, ROW = D * 2, SUB = 32 * ROW;     // 16-byte pieces and bytes of a row, bytes of a sub-tile
    constexpr int COPIES = SUB / 4096;                             // a wavefront's copies (1 KiB each) of a sub-tile
    __shared__ __attribute__((aligned(1024))) uint8_t lds[8 * SUB];       // keys' ring, values' ring
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // heads that share keys go to one XCD (workgroups go around the eight of them)
    int place = blockIdx.x;
    if (place >= 256 && place < a.turned) place = (248 + a.turned - (place & ~7)) | (place & 7);
    int head = place % a.Hq;
    if (a.Hq % 8 == 0) head = (head & 7) * (a.Hq >> 3) + (head >> 3);
    const int kv = head / a.group;
    Tile tl = tile_of(a, place / a.Hq, kRows);
    if (tl.b < 0) return;
    const int ns = splits_of(a, tl);                               // workgroups that share the tile's keys
    if ((int)blockIdx.y >= ns) return;
    const int key0 = blockIdx.y * a.split_steps * 32;              // the first of this one's
    tl.k0 += key0;
    tl.m -= key0;
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
    int seen = a.causal ? min(past + row + 1, tl.m) : tl.m;
    const int last_row = min(tl.n - tl.row, kRows) - 1;            // of the workgroup's rows
    const int all_keys = a.causal ? min(past + tl.row + last_row + 1, tl.m) : tl.m;                                 // that some row sees
    const int wave_last = min(last_row, wave * 32 + 31);
    const int wave_keys = wave * 32 > last_row ? 0 : a.causal ? min(past + tl.row + wave_last + 1, tl.m) : tl.m;    // some row of the wavefront
    const int wave_all = a.causal ? min(past + tl.row + wave * 32 + 1, tl.m) : tl.m;                                // every row of it
    const int there = (max(all_keys, 0) + 31) >> 5;
    const int steps = (int)blockIdx.y == ns - 1 ? there : min(there, a.split_steps);
    const int mine = min((max(wave_keys, 0) + 31) >> 5, steps), whole = min(max(wave_all, 0) >> 5, mine);
    seen = min(seen, steps * 32);                                  // what follows is another workgroup's

    // copies: lane l of a wavefront's copy j brings the piece that belongs at place l of 1 KiB.  Sixteen lanes read LDS at a time,
    // 256 bytes: a row's pieces are permuted by the row so that the sixteen rows (keys) or the four rows of 64 bytes (values) of a
    // read meet every bank once.
    const uint32_t base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds);
    auto key_place = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
    auto value_place = [](int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };
    uint32_t k_off[COPIES], v_off[COPIES];
    auto offsets = [&](uint32_t (&at)[COPIES], int ld, auto place, int rows) {     // rows behind the last one are replaced by it
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            const int r = (wave * COPIES + j) * (64 / PIECES) + lane / PIECES;
            at[j] = (uint32_t)(min(r, rows - 1) * ld + ((lane % PIECES) ^ place(r)) * 8) * 2;
        }
    };
    offsets(k_off, (int)a.ldk, key_place, 32);
    offsets(v_off, (int)a.ldv, value_place, 32);
    const int cut = tl.m % 32 ? tl.m >> 5 : -1;                    // the sub-tile that ends behind the sequence
    const int64_t k_step = a.ldk * 64, v_step = a.ldv * 64;        // bytes
    const uint8_t *k_src = reinterpret_cast<const uint8_t *>(a.k + (int64_t)tl.k0 * a.ldk + kv * D);
    const uint8_t *v_src = reinterpret_cast<const uint8_t *>(a.v + (int64_t)tl.k0 * a.ldv + kv * D);
    int k_next = 0, v_next = 0;                                    // sub-tiles to be copied next
    const uint32_t part = base + wave * (COPIES * 1024);
    auto copy_k = [&] {                                            // behind the last one: the last one again, into a slot nobody reads
        if (k_next == cut) offsets(k_off, (int)a.ldk, key_place, tl.m & 31);
        const uint32_t to = part + (k_next & 3) * SUB;
        lds_dma16_s<0, 0>(k_off[0], k_src, to);
        if constexpr (COPIES == 2) lds_dma16_s<1024, 0>(k_off[COPIES - 1], k_src, to);
        k_src += k_next < steps - 1 ? k_step : 0;
        ++k_next;
    };
    auto copy_v = [&] {
        if (v_next == cut) offsets(v_off, (int)a.ldv, value_place, tl.m & 31);
        const uint32_t to = part + (4 + (v_next & 3)) * SUB;
        lds_dma16_s<0, 0>(v_off[0], v_src, to);
        if constexpr (COPIES == 2) lds_dma16_s<1024, 0>(v_off[COPIES - 1], v_src, to);
        v_src += v_next < steps - 1 ? v_step : 0;
        ++v_next;
    };

    // operand reads: piece 2 st + h of row i; columns 32 d .. + 31 of rows 16 st + 8 e + 4 h .. + 3
    const uint32_t k_lane = base + (uint32_t)(i * ROW) + (uint32_t)((h ^ key_place(i)) << 4);
    const int tr_row = 4 * h + ((lane & 15) >> 2), tr_col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    const uint32_t v_lane = base + 4 * SUB + (uint32_t)(tr_row * ROW) + (uint32_t)(((tr_col >> 3) ^ value_place(tr_row)) << 4) + (tr_col & 7) * 2;
    auto read_k = [&](uint32_t at, int st) { return read_lds(at ^ (uint32_t)(st << 5)); };
    auto read_v = [&](uint32_t at, int d, int st) {
        union {
            short4_t s[2];
            half8_t v;
        } f;
        f.s[0] = read_tr((at ^ (uint32_t)(d << 6)) + st * 16 * ROW);
        f.s[1] = read_tr((at ^ (uint32_t)(d << 6)) + st * 16 * ROW + 8 * ROW);
        return f.v;
    };

    float c = a.scale, off = kNone, l = 0.0f;
    if constexpr (D == 64) asm("" : "+v"(c));                      // a scalar operand takes the ALU half as long again (1 % of D = 64)
    float16_t o[DT], s0 = {}, s1 = {};
    half8_t p0[2] = {}, p1[2] = {};
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = float16_t{};
    const half2_t ones = {(_Float16)1.0f, (_Float16)1.0f};
    auto max3 = [](float x, float y, float z) { return fmaxf(fmaxf(x, y), z); };
    auto top_of = [&](const float16_t &s) {
        const float t0 = max3(s[0], s[1], s[2]), t1 = max3(s[3], s[4], s[5]), t2 = max3(s[6], s[7], s[8]), t3 = max3(s[9], s[10], s[11]);
        const uint32_t x = __float_as_uint(max3(max3(t0, t1, s[15]), max3(t2, t3, s[14]), max3(s[12], s[13], t0)));
        const auto both = __builtin_amdgcn_permlane32_swap(x, x, false, false);      // the other sixteen keys of the query
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    };
    auto weigh = [&](float x0, float x1, half8_t (&p)[2], int g) {   // of scores 2 g and 2 g + 1, their exponents
        const half2_t w = {(_Float16)__builtin_amdgcn_exp2f(x0), (_Float16)__builtin_amdgcn_exp2f(x1)};
        uint32_t bits = __builtin_bit_cast(uint32_t, w);
        asm volatile("" : "+v"(bits));                             // here, beside the matrix instructions, not where p is used
        uint4_t all = __builtin_bit_cast(uint4_t, p[g >> 2]);
        all[g & 3] = bits;
        p[g >> 2] = __builtin_bit_cast(half8_t, all);
        l = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, bits), ones, l, false);
    };

    auto slot = [](int u) { return (uint32_t)(u & 3) * SUB; };

    // the steps that multiply with values under the mask, and what is left at the end
    auto scores = [&](int u, float16_t &s) {
        const uint32_t at = k_lane + slot(u);
        s = float16_t{};
#pragma unroll
        for (int st = 0; st < KS; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_k(at, st), q[st], s, 0, 0, 0);
    };
    auto mask = [&](int u, float16_t &s) {
        const int left = seen - u * 32 - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < left ? s[r] : -INFINITY;
    };
    // Rows with scores of 2^26 and more: the multiply-add of a score and its reference would be off by powers of two, so the
    // reference is a score here, the row's maximum, and is taken off before the scale.
    auto step_plain = [&](int u, auto loud_tag) __attribute__((always_inline)) {                  // scores in s0, probabilities of the sub-tile before in p1
        constexpr bool LOUD = decltype(loud_tag)::value;
        if (u + 1 < mine) scores(u + 1, s1);
        if (u > 0 && u - 1 < mine) {
            const uint32_t at = v_lane + slot(u - 1);
            // values under the mask must not reach the rows that do not see them (0 times an infinity is NaN): infinities and
            // NaN are left out of the product and added where they are seen
            const bool cut = u > whole;
            uint32_t odd = 0;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    half8_t v = read_v(at, d, st);
                    if (cut) {
                        uint4_t w = __builtin_bit_cast(uint4_t, v);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t x = ((w[e] & 0x7C00u) == 0x7C00u ? 0xFFFFu : 0u) | ((w[e] & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u);
                            odd |= x;
                            w[e] &= ~x;
                        }
                        v = __builtin_bit_cast(half8_t, w);
                    }
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p1[st], o[d], 0, 0, 0);
                }
            if (cut && __any(odd)) {
                for (int r = 0; r < 32 && (u - 1) * 32 + r < seen; ++r)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int col = d * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
                            const _Float16 x = *(const __attribute__((address_space(3))) _Float16 *)(uintptr_t)(
                                base + 4 * SUB + slot(u - 1) + r * ROW + (((col >> 3) ^ value_place(r)) << 4) + (col & 7) * 2);
                            if ((__builtin_bit_cast(uint16_t, x) & 0x7C00u) == 0x7C00u) o[d][e] += (float)x;
                        }
            }
        }
        if (u < mine) {
            if (u >= whole) mask(u, s0);
            const float top = top_of(s0), over = LOUD ? top - off : fmaf(top, c, -off);
            if (__any(over > (LOUD ? 0.0f : kSlack + kUpLog2))) {
                const float to = LOUD ? fmaxf(top, off) : over > kSlack + kUpLog2 ? fmaf(top, c, -kUpLog2) : off;
                const float f = __builtin_amdgcn_exp2f(LOUD ? (off - to) * c : off - to);
                off = to;
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= f;
            }
            auto exponent = [&](float x) { return LOUD ? fmaf(x - off, c, kUpLog2) : fmaf(x, c, -off); };
#pragma unroll
            for (int g = 0; g < 8; ++g) weigh(exponent(s0[2 * g]), exponent(s0[2 * g + 1]), p1, g);
        }
        s0 = s1;
    };

    // the others: sub-tile u - 1 seen whole.  (In the first step the weights are 0 and the values those of sub-tile 0; the
    // sums are cleared behind it.  Scores of a sub-tile behind the last one are made and not used.)  The first fragments
    // of a step are read at the end of the one before it (in `fr`) unless the wavefronts meet in between.
    constexpr int AHEAD = 3;
    struct Fragments {
        half8_t k[KS + AHEAD], v[KS + AHEAD];                      // KS == 2 DT: as many products with values
    };
    auto first_reads = [&](int u, Fragments &fr) {
        unroll<AHEAD>([&](auto n) {
            fr.k[n.value] = read_k(k_lane + slot(u + 1), n.value);
            fr.v[n.value] = read_v(v_lane + slot(max(u - 1, 0)), n.value % DT, n.value / DT);
        });
    };
    auto step_full = [&](int u, float16_t &s, float16_t &s_next, half8_t (&p)[2], const half8_t (&p_before)[2], Fragments &fr, auto more_tag, auto mask_tag) {
        constexpr bool MORE = decltype(more_tag)::value, MASK = decltype(mask_tag)::value;     // the next step follows at once; sub-tile u is cut
        const uint32_t at_k = k_lane + slot(u + 1), at_v = v_lane + slot(max(u - 1, 0)), next_k = k_lane + slot(u + 2), next_v = v_lane + slot(u);
        float f = 1.0f, over = 0.0f, top = 0.0f;
        bool raise = false;
        unroll<2 * KS>([&](auto n) {
            constexpr int N = n.value / 2, R = N + AHEAD;
            if constexpr (n.value % 2 == 0) {
                if constexpr (N == 0) s_next = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr.k[0], q[0], float16_t{}, 0, 0, 0);
                else s_next = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr.k[N], q[N], s_next, 0, 0, 0);
                if constexpr (R < KS) fr.k[R] = read_k(at_k, R);
                else if constexpr (MORE) fr.k[R] = read_k(next_k, R - KS);
            } else {
                o[N % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fr.v[N], p_before[N / DT], o[N % DT], 0, 0, 0);
                if constexpr (R < KS) fr.v[R] = read_v(at_v, R % DT, R / DT);
                else if constexpr (MORE) fr.v[R] = read_v(next_v, (R - KS) % DT, (R - KS) / DT);
            }
            // the vector ALU's share: the maximum, the reference, then two scores at a time
            if constexpr (n.value == 0) {
                if constexpr (MASK) mask(u, s);
                top = top_of(s);
            }
            if constexpr (n.value == 1) {
                over = fmaf(top, c, -off);
                raise = __any(over > kSlack + kUpLog2);
                const float to = over > kSlack + kUpLog2 ? fmaf(top, c, -kUpLog2) : off;
                f = __builtin_amdgcn_exp2f(off - to);
                off = to;
                l *= f;
            }
            constexpr int FROM = KS == 8 ? 2 : 1, DONE = (n.value - FROM) * 8 / (2 * KS - 1 - FROM), NEXT = (n.value + 1 - FROM) * 8 / (2 * KS - 1 - FROM);
            if constexpr (n.value >= FROM) {
#pragma unroll
                for (int g = DONE; g < (NEXT < 8 ? NEXT : 8); ++g) weigh(fmaf(s[2 * g], c, -off), fmaf(s[2 * g + 1], c, -off), p, g);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if (MORE && u == 0) {                                      // nothing is summed yet; what the step made of infinities goes
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = float16_t{};
        } else if (raise) {
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= f;                // (an infinity that was seen stays one or becomes NaN, f = 0 or not)
        }
        if constexpr (MORE) unroll<AHEAD>([&](auto n) { fr.k[n.value] = fr.k[KS + n.value], fr.v[n.value] = fr.v[KS + n.value]; });
    };

    if (steps > 0) {
        copy_k();
        copy_k();
        copy_k();
        copy_v();
        meet<2 * COPIES + COPIES>();
        if (mine > 0) scores(0, s0);
        // Whether a row's scores might reach 2^26, by |q| |k| with the largest finite key: half of q is a lane's, so queries of 45 and
        // more in every dimension.
        float square[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const half2_t two = {q[st][2 * e], q[st][2 * e + 1]};
                square[e] = __builtin_amdgcn_fdot2(two, two, square[e], false);
            }
        const bool loud = __any(((square[0] + square[1]) + (square[2] + square[3])) * (c * c) > 0x1p19f / D);
        // Between two pairs of steps: keys' sub-tiles u + 1, u + 2 and values' u - 1, u have landed, and nobody reads the slots
        // any more that the next ones (keys' up to u + 4, values' up to u + 2) get.
        auto turn = [&]() __attribute__((always_inline)) {
            meet<0>();
            copy_k();
            copy_k();
            copy_v();
            copy_v();
        };
        int u = 0;
        auto pair = [&](auto mask_tag) __attribute__((always_inline)) {
            turn();
            Fragments fr;
            first_reads(u, fr);
            step_full(u, s0, s1, p0, p1, fr, std::true_type{}, std::false_type{});
            step_full(u + 1, s1, s0, p1, p0, fr, std::false_type{}, mask_tag);
        };
        auto rest = [&](auto loud_tag) __attribute__((always_inline)) {
            for (; u <= steps; u += 2) {
                turn();
#pragma unroll 1
                for (int e = 0; e < 2; ++e) step_plain(u + e, loud_tag);
            }
        };
        if (__builtin_expect(loud, 0)) {
            rest(std::true_type{});
            off = fmaf(off, c, -kUpLog2);
        } else {
            for (; u + 1 < whole; u += 2) pair(std::false_type{});
            if (u + 1 == whole) {
                pair(std::true_type{});
                u += 2;
            }
            rest(std::false_type{});
        }
        __builtin_amdgcn_s_waitcnt(0x70);                          // the last copies have landed before the LDS is given back
    }
    l += __shfl_xor(l, 32);
    // Out by way of LDS (each wavefront 8 KiB of it, pieces of 16 bytes permuted by the row), so that whole rows are stored: as
    // they lie in the registers, a store would have 16 or 32 bytes of each of 32 rows.
    __syncthreads();
    const uint32_t mine_lds = base + wave * 8192;
    auto rows_out = [&](auto bytes_tag, auto &&store) {
        constexpr int BYTES = decltype(bytes_tag)::value, N = BYTES / 16;      // of a row
        const int r0 = lane / N, p = lane % N;
#pragma unroll
        for (int r = 0; r < 32; r += 64 / N) {
            const uint32_t at = mine_lds + (r + r0) * BYTES + ((p ^ (BYTES == 256 ? (r + r0) & 15 : ((r + r0) >> 1) & 7)) << 4);
            const uint4_t x = *(const __attribute__((address_space(3))) uint4_t *)(uintptr_t)at;
            if (tl.row + wave * 32 + r + r0 < tl.n) store(tl.q0 + tl.row + wave * 32 + r + r0, p, x);
        }
    };
    if (ns > 1) {
        const int64_t at0 = (int64_t)blockIdx.y * a.Tq;
        if (h == 0 && on) a.part_ml[(at0 + tl.q0 + row) * a.Hq + head] = make_float2(off, l);
#pragma unroll
        for (int d = 0; d < DT; d += 2) {
#pragma unroll
            for (int dd = 0; dd < 2; ++dd)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4_t x = {o[d + dd][e * 4], o[d + dd][e * 4 + 1], o[d + dd][e * 4 + 2], o[d + dd][e * 4 + 3]};
                    *(__attribute__((address_space(3))) float4_t *)(uintptr_t)(mine_lds + i * 256 + (((dd * 8 + e * 2 + h) ^ (i & 15)) << 4)) = x;
                }
            rows_out(Int<256>{}, [&](int t, int p, uint4_t x) { *reinterpret_cast<uint4_t *>(a.part + ((at0 + t) * a.Hq + head) * D + d * 32 + p * 4) = x; });
        }
        return;
    }
    const float f = inverse_of(l, seen > 0);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const half2_t lo = {(_Float16)(o[d][e * 4] * f), (_Float16)(o[d][e * 4 + 1] * f)}, hi = {(_Float16)(o[d][e * 4 + 2] * f), (_Float16)(o[d][e * 4 + 3] * f)};
            const uint2_t x = {__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
            *(__attribute__((address_space(3))) uint2_t *)(uintptr_t)(mine_lds + i * ROW + (((d * 4 + e) ^ key_place(i)) << 4) + h * 8) = x;
        }
    rows_out(Int<ROW>{}, [&](int t, int p, uint4_t x) { *reinterpret_cast<uint4_t *>(a.o + (int64_t)t * a.ldo + head * D + p * 8) = x; });
}

// The workgroups of a tile joined: the same tiles and heads, D / 4 lanes to a row, 1024 / D rows to a workgroup.
template <int D>
__global__ __launch_bounds__(256) void attn_packed_join_kernel(const PackedArgs a) {
    constexpr int LANES = D / 4, AHEAD = 8;
    const int head = blockIdx.x % a.Hq;
    const Tile tl = tile_of(a, blockIdx.x / a.Hq, kRows);
    if (tl.b < 0) return;
    const int ns = splits_of(a, tl), r = blockIdx.y * (256 / LANES) + threadIdx.x / LANES;
    if (ns == 1 || tl.row + r >= tl.n) return;
    const int d = threadIdx.x % LANES * 4;
    const int64_t step = (int64_t)a.Tq * a.Hq, t = tl.q0 + tl.row + r, at = t * a.Hq + head;
    float most = kNone, sum = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s = 0; s < ns; s += AHEAD) {
        float2 ml[AHEAD];
        float4 x[AHEAD];
        float to = most;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const int64_t from = at + min(s + e, ns - 1) * step;
            ml[e] = a.part_ml[from];
            x[e] = *reinterpret_cast<const float4 *>(a.part + from * D + d);
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) to = fmaxf(to, ml[e].x);
        const float f0 = __builtin_amdgcn_exp2f(most - to);
        most = to;
        sum *= f0;
        acc.x *= f0, acc.y *= f0, acc.z *= f0, acc.w *= f0;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const bool again = s + e >= ns;                        // the last one's, which may be infinite: not times 0
            const float f = again ? 0.0f : __builtin_amdgcn_exp2f(ml[e].x - to);
            if (again) x[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f), ml[e].y = 0.0f;
            sum = fmaf(ml[e].y, f, sum);
            acc.x = fmaf(x[e].x, f, acc.x), acc.y = fmaf(x[e].y, f, acc.y), acc.z = fmaf(x[e].z, f, acc.z), acc.w = fmaf(x[e].w, f, acc.w);
        }
    }
    const float f = inverse_of(sum, tl.m > 0 && (!a.causal || tl.m - tl.n + tl.row + r >= 0));
    const _Float16 y[4] = {(_Float16)(acc.x * f), (_Float16)(acc.y * f), (_Float16)(acc.z * f), (_Float16)(acc.w * f)};
    *reinterpret_cast<uint2 *>(a.o + t * a.ldo + head * D + d) = __builtin_bit_cast(uint2, y);
}

template <int D>
int launch(PackedArgs a, hipStream_t st) {
    const int64_t tiles = agq_packed_tiles(a.Tq, a.B);
    const unsigned groups = (unsigned)(tiles * a.Hq);
    // One causal prompt: its longest tiles go first, and workgroup n + 256 gets its place on the CU of workgroup n.  So the
    // second 256 are taken in the opposite order (eight at a time, for the XCDs): the longest share a CU with the shortest.
    // Tokens x heads of 128: 4096 x 32 164 -> 157 us, 2048 x 32 54 -> 52, 2500 x 28 65.5 -> 63.7, 6000 x 12 of 64 90 -> 86,
    // 8192 x 32 and longer level; 2048 x 40, where the shortest tiles of all follow, 59.5 -> 60.5 (both sides on one card).
    a.turned = 0;
    if (a.B == 1 && a.causal && a.splits == 1) a.turned = groups < 512 ? (int)groups & ~7 : 512;
    attn_packed_kernel<D><<<dim3(groups, (unsigned)a.splits), 256, 0, st>>>(a);
    const int err = (int)hipGetLastError();
    if (err || a.splits == 1) return err;
    attn_packed_join_kernel<D><<<dim3(groups, kRows * D / 1024), 256, 0, st>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

int agq_launch_attn_packed(const AgqAttnPacked &p, const AgqPackedSplit &sp, void *workspace, void *stream) {
    PackedArgs a;
    a.q = (const _Float16 *)p.q, a.k = (const _Float16 *)p.k, a.v = (const _Float16 *)p.v, a.o = (_Float16 *)p.o;
    a.cu_q = p.cu_q, a.cu_k = p.cu_k;
    a.ldq = p.ldq, a.ldk = p.ldk, a.ldv = p.ldv, a.ldo = p.ldo;
    a.scale = p.scale * 1.44269504088896340736f;
    a.Tq = (int)p.Tq, a.Tk = (int)p.Tk, a.B = (int)p.B, a.Hq = (int)p.Hq, a.group = (int)(p.Hq / p.Hkv), a.causal = p.causal;
    a.splits = sp.splits, a.split_steps = sp.split_steps;
    a.part = (float *)workspace;
    a.part_ml = (float2 *)(a.part + (size_t)a.splits * p.Tq * p.Hq * p.D);
    return p.D == 128 ? launch<128>(a, (hipStream_t)stream) : launch<64>(a, (hipStream_t)stream);
}
