// The paged key/value cache: its book-keeping from the requests' lengths (which pages a step takes and gives back, where
// every new token goes), and the write of a step's keys and values, quantized to 8 bits, into the pages.
#include "agq_device.h"
#include "agq_fp16.h"
#include "agq_internal.h"

namespace {

// ---------------------------------------------------------------- pages, slots and positions of a step
//
// Three prefix sums over the requests: tokens, pages needed, pages given back.  Then every token, every new table entry and
// every returned page is written by itself: its request is found by bisection in the sums.  The free pages are a ring, so
// what a call takes (from the head on) and what it gives back (behind the last free page) are different entries, and no
// workgroup reads what another one writes.  Every workgroup computes the sums by itself, which is less than a launch of
// its own would cost; its share of the tokens and entries is what it writes.  Bound: a launch and the trips
// to memory one after the other (ring state and lengths, table or ring, results): 5.8 us for 256 requests with a token each,
// 5.5 for 40 prompts of up to 2048.
constexpr int kMapThreads = 512;

struct MapArgs {
    const int32_t *kv_len, *n_new, *free_in;
    int32_t *table, *ring, *kv_len_out, *cu_new, *pos, *slot, *free_out, *status;
    int64_t max_pages;
    int B, T, page_log2, n_pages;
};

struct MapRow {      // what one request asks for
    int64_t tokens, need, back;
    int past, held;
    bool bad, gone;
};
__device__ __forceinline__ MapRow map_row(int past, int add, int page_log2, int64_t capacity) {
    const int64_t page1 = ((int64_t)1 << page_log2) - 1;
    MapRow r;
    const int64_t after = (int64_t)past + max(add, 0);
    r.bad = past < 0 || add < -1 || after > capacity;
    const int64_t held = (past + page1) >> page_log2;
    r.past = past;
    r.gone = add < 0;
    r.held = (int)held;
    r.tokens = r.bad ? 0 : max(add, 0);
    r.need = r.bad || add <= 0 ? 0 : ((after + page1) >> page_log2) - held;
    r.back = r.bad || add >= 0 ? 0 : held;
    return r;
}

__global__ __launch_bounds__(kMapThreads) void kv_map_kernel(const MapArgs a) {
    __shared__ int64_t sums[3][kMapThreads / 64];
    __shared__ int bad_wave[kMapThreads / 64];
    __shared__ int at_tok[kMapThreads], at_need[kMapThreads], at_back[kMapThreads], past_of[kMapThreads], held_of[kMapThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t capacity = a.max_pages << a.page_log2;
    const int head = a.free_in[0], count = a.free_in[1];
    // Sums over a batch of kMapThreads requests: every thread's own and what is before it, the totals in `sums` (64 bits: a
    // request may ask for anything), by scans of the halves of 32-bit numbers.
    struct Mine {
        int64_t tok, need, back;
    };
    auto scan64 = [&](int64_t v) { return ((int64_t)agq_wave_scan((int)(v >> 16)) << 16) + agq_wave_scan((int)(v & 0xFFFF)); };
    auto batch = [&](const MapRow &r, bool bad) {
        const Mine up = {scan64(r.tokens), scan64(r.need), scan64(r.back)};
        const int any_bad = __any(bad);
        __syncthreads();
        if (lane == 63) sums[0][wave] = up.tok, sums[1][wave] = up.need, sums[2][wave] = up.back, bad_wave[wave] = any_bad;
        __syncthreads();
        return Mine{up.tok - r.tokens, up.need - r.need, up.back - r.back};
    };
    auto row_of = [&](int b) { return b < a.B ? map_row(a.kv_len[b], a.n_new[b], a.page_log2, capacity) : MapRow{}; };
    // the totals, and whether the step can be done at all
    int64_t tokens = 0, need = 0, back = 0;
    bool bad = head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages;
    MapRow r = row_of(tid);
    Mine before = batch(r, r.bad);
    for (int b0 = 0;;) {
#pragma unroll
        for (int w = 0; w < kMapThreads / 64; ++w) tokens += sums[0][w], need += sums[1][w], back += sums[2][w], bad |= bad_wave[w] != 0;
        if ((b0 += kMapThreads) >= a.B) break;
        const MapRow more = row_of(b0 + tid);
        batch(more, more.bad);
    }
    bad |= tokens > a.T || count + back > a.n_pages;
    const bool go = !bad && need <= count;
    const bool first = blockIdx.x == 0;
    auto ring_at = [&](int64_t i) {                          // i < 2 n_pages
        const uint32_t at = (uint32_t)head + (uint32_t)i;
        return (int)(at >= (uint32_t)a.n_pages ? at - (uint32_t)a.n_pages : at);
    };
    if (first && tid == 0) {
        const int64_t missing = min(need - count, (int64_t)0x7FFFFFFF);
        *a.status = bad ? -1 : go ? 0 : (int)missing;
        a.free_out[0] = go ? ring_at(need) : head;
        a.free_out[1] = go ? (int)(count - need + back) : count;
        a.cu_new[0] = 0;
    }
    const int per = (a.T + gridDim.x - 1) / gridDim.x;      // this workgroup's tokens
    const int t0 = min((int64_t)blockIdx.x * per, (int64_t)a.T), t1 = min(t0 + per, a.T);
    if (!go) {
        for (int t = t0 + tid; t < t1; t += kMapThreads) a.pos[t] = 0, a.slot[t] = -1;
        if (first)
            for (int b = tid; b < a.B; b += kMapThreads) a.kv_len_out[b] = a.kv_len[b], a.cu_new[b + 1] = 0;
        return;
    }
    for (int t = max(t0, (int)tokens) + tid; t < t1; t += kMapThreads) a.pos[t] = 0, a.slot[t] = -1;
    const int per_need = ((int)need + gridDim.x - 1) / gridDim.x, per_back = ((int)back + gridDim.x - 1) / gridDim.x;
    const int n0 = min((int64_t)blockIdx.x * per_need, need), n1 = min(n0 + per_need, (int)need);
    const int k0 = min((int64_t)blockIdx.x * per_back, back), k1 = min(k0 + per_back, (int)back);

    int done_tok = 0, done_need = 0, done_back = 0;          // sums of the requests before this batch; they fit now
    for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
        const int b = b0 + tid, n = min(kMapThreads, a.B - b0);
        if (a.B > kMapThreads) {                             // one batch: its sums are still there
            r = row_of(b);
            before = batch(r, false);
        }
        int e_tok = done_tok + (int)before.tok, e_need = done_need + (int)before.need, e_back = done_back + (int)before.back;
#pragma unroll
        for (int w = 0; w < kMapThreads / 64; ++w) {
            const int x = (int)sums[0][w], y = (int)sums[1][w], z = (int)sums[2][w];
            if (w < wave) e_tok += x, e_need += y, e_back += z;
            done_tok += x, done_need += y, done_back += z;
        }
        at_tok[tid] = e_tok, at_need[tid] = e_need, at_back[tid] = e_back, past_of[tid] = r.past, held_of[tid] = r.held;
        if (first && b < a.B) {
            a.cu_new[b + 1] = e_tok + (int)r.tokens;
            a.kv_len_out[b] = r.gone ? 0 : r.past + (int)r.tokens;
        }
        __syncthreads();
        // the tokens of these requests that are this workgroup's
        for (int t = max(t0, at_tok[0]) + tid; t < min(t1, done_tok); t += kMapThreads) {
            const int i = agq_find_row(at_tok, n, t);
            const int p = past_of[i] + t - at_tok[i], j = p >> a.page_log2;
            const int id = j < held_of[i] ? a.table[(int64_t)(b0 + i) * a.max_pages + j] : a.ring[ring_at((int64_t)at_need[i] + j - held_of[i])];
            a.pos[t] = p;
            a.slot[t] = (unsigned)id < (unsigned)a.n_pages ? (id << a.page_log2) + (p & ((1 << a.page_log2) - 1)) : -1;
        }
        for (int u = max(n0, at_need[0]) + tid; u < min(n1, done_need); u += kMapThreads) {
            const int i = agq_find_row(at_need, n, u);
            a.table[(int64_t)(b0 + i) * a.max_pages + held_of[i] + u - at_need[i]] = a.ring[ring_at(u)];
        }
        for (int u = max(k0, at_back[0]) + tid; u < min(k1, done_back); u += kMapThreads) {
            const int i = agq_find_row(at_back, n, u);
            a.ring[ring_at((int64_t)count + u)] = a.table[(int64_t)(b0 + i) * a.max_pages + u - at_back[i]];
        }
    }
}

// ---------------------------------------------------------------- rotary embedding, Eq.2 into the pages
//
// A run is the tokens of the call that lie one behind the other in one page; it is done in one piece, for one head, keys or
// values.  The scale of a page and head is the smallest power of two that clips nothing (agq_calibrate_act_exp's rule) over
// the run, and not below the one that the page's earlier tokens have: those are divided by what it grew by, halves to the
// even code.  Keys lie [token, D] in a page; values [D, token], which is the order in which the attention's matrix
// instructions take them, so it reads both straight into registers.
// The rotation is float64, in which products of fp16 and fp32 numbers are exact, rounded once.  Bound: long runs by memory and
// the float64 arithmetic beside it (6000 tokens of 40 heads of 128: 372 MB in 96 us, 3.9 TB/s; a copy reaches 4.9),
// a step's tokens by latency (one of 32 heads 4.3 us, 256 of 32 query and 8 key heads 8.0: 12.0 MB written for
// 3.1, as a token's values are a byte in each of D rows).
struct AppendArgs {
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;
    int64_t ldq, ldk, ldv, ldqo, ldko;
    const int32_t *pos, *slot;
    const float *cos_t, *sin_t;
    int8_t *kc, *vc, *ke, *ve;
    int T, Hq, Hkv, D, D_log2, P, page, page_log2, n_pages, chunk, chunks;
    // normalised heads: gains [D] of head h at g + h * ldg
    const uint16_t *g_q, *g_k;
    int64_t ldgq, ldgk;
    double eps;
    int q_apart;                 // groups of lanes for a token's queries
};
constexpr int kEZero = -30;      // the smallest exponent that a nonzero fp16 value asks for; pages of zeros get it too

// the smallest e with top <= 127 * 2^e, top the bits of a nonnegative fp16 value (infinity counts as 2^16)
__device__ __forceinline__ int exp_for(uint32_t top) {
    if (top == 0) return kEZero;
    const float f = top >= 0x7C00u ? 65536.0f : __half2float(__ushort_as_half((uint16_t)top));
    const uint32_t u = __float_as_uint(f);                       // fp16 values are normal in fp32
    const int x = (int)(u >> 23) - 127;                          // f = m 2^x, 1 <= m < 2
    return (u & 0x7FFFFFu) <= 0x7E0000u ? x - 6 : x - 5;         // m <= 127 / 64
}

// float64 -> fp16 as in d2h, by way of the twenty leading bits of the fraction: any bit behind them sets the last one (rounding
// to odd), which the one rounding that follows sees; they are exact in fp32.
__device__ __forceinline__ uint16_t d2h_odd(double d) {
    const uint64_t u = __builtin_bit_cast(uint64_t, d);
    const uint32_t hi = (uint32_t)(u >> 32) | min((uint32_t)u, 1u);
    float f = (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
    asm("" : "+v"(f));                  // else the compiler makes one conversion of the two, of some thirty instructions
    return __half_as_ushort(__float2half_rn(f));
}
// eight pairs of a head turned by their angles
__device__ __forceinline__ void rotate8(Half8 &lo, Half8 &hi, const float *cos_t, const float *sin_t) {
    const float4 c0 = reinterpret_cast<const float4 *>(cos_t)[0], c1 = reinterpret_cast<const float4 *>(cos_t)[1];
    const float4 s0 = reinterpret_cast<const float4 *>(sin_t)[0], s1 = reinterpret_cast<const float4 *>(sin_t)[1];
    const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double l = h2d(lo.v[i]), h = h2d(hi.v[i]), c = (double)cs[i], s = (double)sn[i];
        lo.v[i] = d2h_odd(l * c - h * s);
        hi.v[i] = d2h_odd(h * c + l * s);
    }
}
// 1 / sqrt(a) to float64's last bit or two: the instruction's 2^-26 or better, and y += y (1 - a y^2) / 2 twice.  Infinite
// for 0, and 0 for infinity, as the quotient would be.
__device__ __forceinline__ double inv_sqrt(double a) {
    const double y = __builtin_amdgcn_rsq(a);
    double r = fma(y, 0.5 * fma(-a * y, y, 1.0), y);
    r = fma(r, 0.5 * fma(-a * r, r, 1.0), r);
    return a > 0.0 && a < __builtin_inf() ? r : y;
}
// What a lane does to its eight pairs of a head, y = inv (l a - h b), inv (h c + l d): gains and angles are multiplied once for
// all heads that have them (exactly: 11 and 24 bits).  Without a rotation l and h stay apart: y = inv l a, inv h c.
struct Turn {
    double a[8], b[8], c[8], d[8];
};
template <bool ROPE>
__device__ __forceinline__ Turn turn_of(const uint16_t *gain, int Dh, const float *cos_t, const float *sin_t) {
    Half8 gl, gh;
    if (gain) {
        gl = load8(gain), gh = load8(gain + Dh);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) gl.v[i] = gh.v[i] = 0x3C00;          // 1
    }
    Turn t;
    if constexpr (ROPE) {
        const float4 c0 = reinterpret_cast<const float4 *>(cos_t)[0], c1 = reinterpret_cast<const float4 *>(cos_t)[1];
        const float4 s0 = reinterpret_cast<const float4 *>(sin_t)[0], s1 = reinterpret_cast<const float4 *>(sin_t)[1];
        const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
        const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double l = h2d(gl.v[i]), h = h2d(gh.v[i]), c = (double)cs[i], n = (double)sn[i];
            t.a[i] = l * c, t.b[i] = h * n, t.c[i] = h * c, t.d[i] = l * n;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) t.a[i] = h2d(gl.v[i]), t.c[i] = h2d(gh.v[i]);
    }
    return t;
}
// The head's other pairs are the neighbouring lanes' (2^per_log2 of them, all active): their squares are summed across them in
// pairs, so every lane has the same sum whatever its place.  norm false: inv = 1.
template <bool ROPE>
__device__ __forceinline__ void turn8(Half8 &lo, Half8 &hi, const Turn &t, bool norm, int Dh, int per_log2, double eps) {
    double inv = 1.0;
    if (norm) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double l = h2d(lo.v[i]), h = h2d(hi.v[i]);
            sum = fma(h, h, fma(l, l, sum));
        }
        for (int m = 1; m < 1 << per_log2; m <<= 1) sum += __shfl_xor(sum, m);
        inv = inv_sqrt(sum * (Dh == 64 ? 1.0 / 128 : 1.0 / 64) + eps);
    }
    // widened a second time: held in float64 they would take 32 registers, and a SIMD three wavefronts instead of four
    asm("" : "+v"(*reinterpret_cast<agq_v4i *>(&lo)), "+v"(*reinterpret_cast<agq_v4i *>(&hi)));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double l = h2d(lo.v[i]), h = h2d(hi.v[i]);
        lo.v[i] = d2h_odd(ROPE ? inv * fma(l, t.a[i], -(h * t.b[i])) : inv * (l * t.a[i]));
        hi.v[i] = d2h_odd(ROPE ? inv * fma(h, t.c[i], l * t.d[i]) : inv * (h * t.c[i]));
    }
}
// The same for one head by itself, whose gains and angles nothing else uses (fewer registers).
template <bool ROPE>
__device__ __forceinline__ void turn8_once(Half8 &lo, Half8 &hi, const uint16_t *gain, int Dh, int per_log2, double eps, const float *cos_t, const float *sin_t) {
    Half8 gl = load8(gain), gh = load8(gain + Dh);
    float cs[8], sn[8];
    if constexpr (ROPE) {
        __builtin_memcpy(cs, cos_t, 32);
        __builtin_memcpy(sn, sin_t, 32);
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double l = h2d(lo.v[i]), h = h2d(hi.v[i]);
        sum = fma(h, h, fma(l, l, sum));
    }
    for (int m = 1; m < 1 << per_log2; m <<= 1) sum += __shfl_xor(sum, m);
    const double inv = inv_sqrt(sum * (Dh == 64 ? 1.0 / 128 : 1.0 / 64) + eps);
    asm("" : "+v"(*reinterpret_cast<agq_v4i *>(&lo)), "+v"(*reinterpret_cast<agq_v4i *>(&hi)));          // widened a second time, as in turn8
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double l = h2d(lo.v[i]) * h2d(gl.v[i]), h = h2d(hi.v[i]) * h2d(gh.v[i]);           // exact
        if constexpr (ROPE) {
            const double c = (double)cs[i], n = (double)sn[i];
            lo.v[i] = d2h_odd(inv * fma(l, c, -(h * n)));
            hi.v[i] = d2h_odd(inv * fma(h, c, l * n));
        } else {
            lo.v[i] = d2h_odd(inv * l), hi.v[i] = d2h_odd(inv * h);
        }
    }
}
// Some heads of one token by the 2^per_log2 lanes of a head: first, first + apart, and so on.
struct Heads {
    const uint16_t *src, *gain;          // of the token; gain NULL: no norm
    uint16_t *dst;
    int64_t ldg;                         // 0: one gain for all heads
    int heads, apart, D;
};
template <bool ROPE>
__device__ __forceinline__ void turn_heads(const Heads &a, int first, const float *cos_t, const float *sin_t, int per_log2, double eps, int lane) {
    const int Dh = a.D >> 1, j = (lane & ((1 << per_log2) - 1)) * 8;
    Turn t = turn_of<ROPE>(a.gain ? a.gain + first * a.ldg + j : nullptr, Dh, cos_t + j, sin_t + j);
    Half8 lo = load8(a.src + first * a.D + j), hi = load8(a.src + first * a.D + j + Dh);
    for (int h = first; h < a.heads; h += a.apart) {
        Half8 x = lo, y = hi;
        if (h + a.apart < a.heads) lo = load8(a.src + (h + a.apart) * a.D + j), hi = load8(a.src + (h + a.apart) * a.D + j + Dh);
        if (h > first && a.ldg != 0) t = turn_of<ROPE>(a.gain + h * a.ldg + j, Dh, cos_t + j, sin_t + j);
        turn8<ROPE>(x, y, t, a.gain != nullptr, Dh, per_log2, eps);
        store8(a.dst + h * a.D + j, x);
        store8(a.dst + h * a.D + j + Dh, y);
    }
}
// the largest magnitude of eight fp16 values, as bits; NaN does not count
__device__ __forceinline__ uint32_t top8(const Half8 &h) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = h.v[i] & 0x7FFFu;
        m = max(m, b > 0x7C00u ? 0u : b);
    }
    return m;
}

// One run: n tokens from t on into the page `id`, its entries off .. off + n - 1, keys (role 2 h) or values (2 h + 1) of head h.
// ALONE: a few tokens, by one wavefront, which has at most one work item per lane; else by the whole workgroup, and the
// fp16 values wait in LDS for the scale.  A work item is eight pairs of a key, or eight of a value.
template <bool ALONE, bool NORM>
__device__ __forceinline__ void append_run(const AppendArgs &a, int role, int t, int n, int64_t id, int off, int tid, int threads, uint16_t *held) {
    const bool values = role & 1;
    const int head = role >> 1, Dh = a.D >> 1, per_log2 = a.D_log2 - (values ? 3 : 4), items = n << per_log2, lane = tid & 63;
    const uint16_t *src = values ? a.v + (int64_t)t * a.ldv + head * a.D : a.k + (int64_t)t * a.ldk + head * a.D;
    const int64_t ld = values ? a.ldv : a.ldk;
    int8_t *e_at = (values ? a.ve : a.ke) + id * a.Hkv + head;
    const int e_had = off ? *e_at : -128;
    uint32_t *tops = reinterpret_cast<uint32_t *>(held + ((size_t)a.page << a.D_log2));
    Half8 lo, hi;
    uint32_t top = 0;
    if (!ALONE) __syncthreads();              // the run before is done with the LDS
    for (int it = tid; it < items; it += threads) {
        const int i = it >> per_log2, j = (it & ((1 << per_log2) - 1)) * 8;
        lo = load8(src + i * ld + j);
        if (!values) {
            hi = load8(src + i * ld + j + Dh);
            const int64_t p = a.cos_t ? min(max(a.pos[t + i], 0), a.P - 1) : 0;
            if constexpr (NORM) {
                const uint16_t *gain = a.g_k + head * a.ldgk + j;
                if (a.cos_t)
                    turn8_once<true>(lo, hi, gain, Dh, per_log2, a.eps, a.cos_t + p * Dh + j, a.sin_t + p * Dh + j);
                else
                    turn8_once<false>(lo, hi, gain, Dh, per_log2, a.eps, nullptr, nullptr);
            } else if (a.cos_t)
                rotate8(lo, hi, a.cos_t + p * Dh + j, a.sin_t + p * Dh + j);
            if (a.k_out) {
                uint16_t *dst = a.k_out + (int64_t)(t + i) * a.ldko + head * a.D + j;
                store8(dst, lo);
                store8(dst + Dh, hi);
            }
            top = max(top, top8(hi));
            if (!ALONE) store8(held + (i << a.D_log2) + j + Dh, hi);
        }
        top = max(top, top8(lo));
        if (!ALONE) store8(held + (i << a.D_log2) + j, lo);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (!ALONE) {
        if (lane == 0) tops[tid >> 6] = top;
        __syncthreads();
        for (int w = 0; w < threads >> 6; ++w) top = max(top, tops[w]);
    }
    const int e = max(exp_for(top), e_had);
    const float inv = __builtin_amdgcn_ldexpf(1.0f, -e);
    const float down = __builtin_amdgcn_ldexpf(1.0f, e_had - e);
    const AgqQuant eq2 = {inv, AGQ_MAGIC - 128.0f, AGQ_MAGIC + 127.0f, 0, 0, 0, 0, 0};
    if (tid == 0) *e_at = (int8_t)e;
    int8_t *codes = (values ? a.vc : a.kc) + ((id * a.Hkv + head) << (a.page_log2 + a.D_log2));
    if (!values) {
        if (off && e > e_had)
            for (int w = tid; w < off << (a.D_log2 - 2); w += threads) {
                uint32_t *p = reinterpret_cast<uint32_t *>(codes) + w;
                *p = agq_coarser4(*p, down);
            }
        if (ALONE) {
            if (tid < items) {
                int8_t *dst = codes + ((off + (tid >> per_log2)) << a.D_log2) + (tid & ((1 << per_log2) - 1)) * 8;
                *reinterpret_cast<uint2 *>(dst) = agq_quant8(__builtin_bit_cast(uint4, lo), eq2);
                *reinterpret_cast<uint2 *>(dst + Dh) = agq_quant8(__builtin_bit_cast(uint4, hi), eq2);
            }
        } else {
            for (int w = tid; w < n << (a.D_log2 - 3); w += threads)
                *reinterpret_cast<uint2 *>(codes + (off << a.D_log2) + w * 8) = agq_quant8(*reinterpret_cast<const uint4 *>(held + w * 8), eq2);
        }
        return;
    }
    // A thread: sixteen tokens of one row (d), lanes along d: one store where all of them are the run's; else in words and
    // bytes, so that only the run's are touched, and older ones if their scale changed.
    const int w0 = e > e_had && off ? 0 : off >> 4, w1 = (off + n + 15) >> 4;
    for (int it = tid; it < (w1 - w0) << a.D_log2; it += threads) {
        const int d = it & (a.D - 1), w = w0 + (it >> a.D_log2), first = w * 16 - off;       // the first of the sixteen in the run
        int8_t *p = codes + (d << a.page_log2) + w * 16;
        auto code = [&](int i) {
            const uint16_t x = ALONE ? src[(first + i) * ld + d] : held[((first + i) << a.D_log2) + d];
            return agq_quant1(__half2float(__ushort_as_half(x)), eq2);
        };
        if (!ALONE && first >= 0 && first + 16 <= n) {
            uint32_t c[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = code(i);
            *reinterpret_cast<uint4 *>(p) = make_uint4(agq_pack4(c[0], c[1], c[2], c[3]), agq_pack4(c[4], c[5], c[6], c[7]),
                                                       agq_pack4(c[8], c[9], c[10], c[11]), agq_pack4(c[12], c[13], c[14], c[15]));
            continue;
        }
        if (first < 0 && e > e_had)
#pragma unroll 1
            for (int j = 0; j < min(-first, 16); ++j) p[j] = agq_coarser(p[j], down);
#pragma unroll 1
        for (int j = max(-first, 0); j < min(n - first, 16); ++j) p[j] = (int8_t)code(j);
    }
}

// ROLES = 1: a workgroup takes the runs that begin in its chunk of tokens, for one role (the keys or the values of a head).
// ROLES = 4: one token and four roles to a workgroup.  A short run, as in a generation step, is that of its first token's
// workgroup, whose wavefronts have a role each; a long one is shared by the workgroups of its first four tokens, a role each.
// NORM: queries and keys are normalised before their rotation; a step's five workgroups of a CU are to fit it (256 tokens of 32 query
// and 8 key heads 9.5 -> 8.9 us).  7001 normalised tokens of 32 and 8 heads of 64: 88 MB in 24 us, 3.6 TB/s.
template <int ROLES, bool NORM>
__global__ __launch_bounds__(256, NORM && ROLES == 4 ? 6 : 1) void kv_append_kernel(const AppendArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint16_t held[];      // [run][D], then one word per wavefront
    const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slots = a.n_pages << a.page_log2, roles = 2 * a.Hkv, groups = (roles + ROLES - 1) / ROLES;
    const unsigned kv_groups = a.chunks * groups;
    if (blockIdx.x >= kv_groups) {                                       // queries: nothing to store but themselves
        const int per_log2 = a.D_log2 - 4, Dh = a.D >> 1;
        if constexpr (NORM && ROLES == 1) {                              // q_apart groups of lanes to a token
            const unsigned group = ((blockIdx.x - kv_groups) * threads + tid) >> per_log2;
            const int t = (int)(group / (unsigned)a.q_apart), first = (int)group - t * a.q_apart;
            if (t >= a.T || (unsigned)a.slot[t] >= (unsigned)slots) return;
            const Heads h = {a.q + (int64_t)t * a.ldq, a.g_q, a.q_out + (int64_t)t * a.ldqo, a.ldgq, a.Hq, a.q_apart, a.D};
            if (a.cos_t) {
                const int64_t p = min(max(a.pos[t], 0), a.P - 1);
                turn_heads<true>(h, first, a.cos_t + p * Dh, a.sin_t + p * Dh, per_log2, a.eps, lane);
            } else {
                turn_heads<false>(h, first, nullptr, nullptr, per_log2, a.eps, lane);
            }
            return;
        }
        const unsigned item = (blockIdx.x - kv_groups) * threads + tid, th = item >> per_log2;   // below 2^31 (the caller's check)
        const int t = (int)(th / (unsigned)a.Hq), h = (int)th - t * a.Hq, j = (int)(item & ((1u << per_log2) - 1)) * 8;
        if (t >= a.T || (unsigned)a.slot[t] >= (unsigned)slots) return;
        const uint16_t *src = a.q + (int64_t)t * a.ldq + h * a.D + j;
        uint16_t *dst = a.q_out + (int64_t)t * a.ldqo + h * a.D + j;
        Half8 lo = load8(src), hi = load8(src + Dh);
        const int64_t p = NORM && !a.cos_t ? 0 : min(max(a.pos[t], 0), a.P - 1);
        if constexpr (NORM) {
            if (a.cos_t)
                turn8_once<true>(lo, hi, a.g_q + h * a.ldgq + j, Dh, per_log2, a.eps, a.cos_t + p * Dh + j, a.sin_t + p * Dh + j);
            else
                turn8_once<false>(lo, hi, a.g_q + h * a.ldgq + j, Dh, per_log2, a.eps, nullptr, nullptr);
        } else {
            rotate8(lo, hi, a.cos_t + p * Dh + j, a.sin_t + p * Dh + j);
        }
        store8(dst, lo);
        store8(dst + Dh, hi);
        return;
    }
    const int c0 = (int)(blockIdx.x / groups) * a.chunk, role0 = (int)(blockIdx.x % groups) * ROLES, end = min(c0 + a.chunk, a.T);
    const int page1 = a.page - 1;
    if constexpr (ROLES == 4) {
        const int u = c0 - 4 + lane, s = u >= 0 && u < a.T ? a.slot[u] : -1, sl = __builtin_amdgcn_readlane(s, 4), off = sl & page1;
        if ((unsigned)sl >= (unsigned)slots) return;
        // tokens of the run before this one (up to four are looked at), and from it on
        const unsigned long long joined = __ballot(s == sl + lane - 4 && off + lane - 4 >= 0 && off + lane - 4 < a.page);
        const int before = __clz(~((unsigned)joined << 28));
        if (before == 4) return;
        int n = before + __ffsll((long long)~(joined >> 4)) - 1;         // sixty of them at most
        for (bool more = n == before + 60; more;) {
            const int i = n - before + lane;
            const bool goes_on = c0 + i < a.T && off + i < a.page && a.slot[min(c0 + i, a.T - 1)] == sl + i;
            const unsigned long long m = __ballot(!goes_on);
            n += m ? __ffsll((long long)m) - 1 : 64;
            more = m == 0;
        }
        const int64_t id = sl >> a.page_log2;
        const int t = c0 - before, role = role0 + (n << (a.D_log2 - 3) <= 64 ? wave : before);
        if (role >= roles) return;
        if (n << (a.D_log2 - 3) <= 64) {
            if (before == 0) append_run<true, NORM>(a, role, t, n, id, off, lane, 64, held);
        } else {
            append_run<false, NORM>(a, role, t, n, id, off - before, tid, threads, held);
        }
        return;
    }
    for (int t = c0; t < end;) {
        // the next token from t on that begins a run
        int sl = -1;
        for (; t < end; t += 64) {
            const int u = t + lane;
            int s = -1;
            bool begins = false;
            if (u < end) {
                s = a.slot[u];
                const int before = u > 0 ? a.slot[u - 1] : -1;
                begins = (unsigned)s < (unsigned)slots && ((s & page1) == 0 || before != s - 1);
            }
            const unsigned long long m = __ballot(begins);
            if (m) {
                const int i = __ffsll((long long)m) - 1;
                sl = __builtin_amdgcn_readlane(s, i);
                t += i;
                break;
            }
        }
        if (t >= end) break;
        const int off = sl & page1;
        const int64_t id = sl >> a.page_log2;
        int n = 1;
        for (;;) {
            const int i = n + lane;
            const bool goes_on = t + i < a.T && off + i < a.page && a.slot[min(t + i, a.T - 1)] == sl + i;
            const unsigned long long m = __ballot(!goes_on);
            if (m) {
                n += __ffsll((long long)m) - 1;
                break;
            }
            n += 64;
        }
        if (n << (a.D_log2 - 3) <= 64) {
            if (wave == 0) append_run<true, NORM>(a, role0, t, n, id, off, lane, 64, held);
        } else {
            append_run<false, NORM>(a, role0, t, n, id, off, tid, threads, held);
        }
        t += n;
    }
}

// ---------------------------------------------------------------- normalised and rotated heads, fp16 to fp16
//
// y = (x r) g rotated by the token's angles, r = 1 / sqrt(mean of x^2 + eps) of the head: float64 throughout, one rounding to fp16.
// A lane has sixteen values of a head, eight of each half, which the rotation brings together; the sum of squares is joined over
// the D / 16 lanes of the head.  They take some heads of one token, of q or of k, one after the other, so that the token's angles
// and the gains are read and multiplied once for them.  Bound: long prompts by memory (6000 tokens of 40 query and 40 key heads of
// 128: 249 MB in 55 us, 4.5 TB/s, a copy reaches 4.8); one token of 32 and 32 heads by latency, 3.2 us.  (Stores past the caches
// take 51, but the attention that reads the results comes next: both together 153 -> 158.)
struct HeadsArgs {
    const uint16_t *q, *k, *g_q, *g_k;
    uint16_t *q_out, *k_out;
    int64_t ldq, ldk, ldgq, ldgk, ldqo, ldko;
    const int32_t *pos;
    const float *cos_t, *sin_t;
    double eps;
    int T, Hq, Hkv, D, per_log2, P, q_apart, k_apart;            // groups of lanes for a token's queries and keys
};
template <bool ROPE>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const HeadsArgs a) {
    const int lane = threadIdx.x & 63, apart = a.q_apart + a.k_apart, Dh = a.D >> 1;
    const unsigned group = (blockIdx.x * 256u + threadIdx.x) >> a.per_log2;                              // below 2^31
    const int t = (int)(group / (unsigned)apart), part = (int)group - t * apart;
    if (t >= a.T) return;
    const bool keys = part >= a.q_apart;
    const Heads h = {keys ? a.k + (int64_t)t * a.ldk : a.q + (int64_t)t * a.ldq, keys ? a.g_k : a.g_q,
                     keys ? a.k_out + (int64_t)t * a.ldko : a.q_out + (int64_t)t * a.ldqo, keys ? a.ldgk : a.ldgq, keys ? a.Hkv : a.Hq,
                     keys ? a.k_apart : a.q_apart, a.D};
    const int64_t p = ROPE ? min(max(a.pos[t], 0), a.P - 1) : 0;
    turn_heads<ROPE>(h, keys ? part - a.q_apart : part, a.cos_t + p * Dh, a.sin_t + p * Dh, a.per_log2, a.eps, lane);
}

}  // namespace

static int log2_of(int64_t v) { return __builtin_ctzll((unsigned long long)v); }
// Groups of lanes for the heads of a token: up to eight heads to each, as long as about 4096 wavefronts are left in all.
static int apart_of(int64_t heads, int64_t all_heads, int64_t T, int64_t D) {
    const int64_t most = T * all_heads * (D / 16) / (4096 * 64), times = most < 1 ? 1 : most > 8 ? 8 : most;
    return (int)((heads + times - 1) / times);
}

int agq_launch_kv_map(const int32_t *kv_len, const int32_t *n_new, int64_t B, int page, int32_t *block_table, int64_t max_pages,
                      int32_t *free_ring, int64_t n_pages, const int32_t *free_state, int64_t T, int32_t *kv_len_out, int32_t *cu_new,
                      int32_t *pos, int32_t *slot, int32_t *free_state_out, int32_t *status, void *stream) {
    const MapArgs a = {kv_len, n_new, free_state, block_table, free_ring, kv_len_out, cu_new, pos, slot, free_state_out, status,
                       max_pages, (int)B, (int)T, log2_of(page), (int)n_pages};
    const int64_t groups = (T + 2 * kMapThreads - 1) / (2 * kMapThreads);
    kv_map_kernel<<<dim3((unsigned)(groups < 1 ? 1 : groups > 256 ? 256 : groups)), kMapThreads, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

int agq_launch_kv_append(const AgqKvAppend &p, void *stream) {
    AppendArgs a;
    a.q = (const uint16_t *)p.q, a.k = (const uint16_t *)p.k, a.v = (const uint16_t *)p.v;
    a.q_out = (uint16_t *)p.q_out, a.k_out = (uint16_t *)p.k_out;
    a.ldq = p.ldq, a.ldk = p.ldk, a.ldv = p.ldv, a.ldqo = p.ldqo, a.ldko = p.ldko;
    a.pos = p.pos, a.slot = p.slot, a.cos_t = p.rope_cos, a.sin_t = p.rope_sin;
    a.kc = p.k_cache, a.vc = p.v_cache, a.ke = p.k_exp, a.ve = p.v_exp;
    a.g_q = (const uint16_t *)p.g_q, a.g_k = (const uint16_t *)p.g_k, a.ldgq = p.ldgq, a.ldgk = p.ldgk, a.eps = p.eps;
    a.T = (int)p.T, a.Hq = (int)p.Hq, a.Hkv = (int)p.Hkv, a.D = (int)p.D, a.D_log2 = log2_of(p.D), a.P = (int)p.P;
    a.page = p.page, a.page_log2 = log2_of(p.page), a.n_pages = (int)p.n_pages;
    // Chunks: a run of a whole page or more to a workgroup, as those that find none to begin take turns with the others (6000
    // tokens, 8 heads of keys, pages of 64: chunks of 8, 32 and 64 tokens 29, 19.5 and 18.8 us).  Four roles: up to 8192
    // workgroups (256 tokens of 32 heads 29.7 -> 18.5 us, 256 of 8 heads 12.7 -> 8.0, one of 32 heads 4.45 -> 4.25 against one
    // role and 64 threads a workgroup).
    const int roles = p.T * 2 * p.Hkv <= 32768 ? 4 : 1;
    int chunk = 1;
    while (roles == 1 && chunk < 128 && p.T * 2 * p.Hkv > (int64_t)chunk * 2048) chunk *= 2;
    a.chunk = chunk;
    a.chunks = (int)((p.T + chunk - 1) / chunk);
    // one item of a full page's keys to a thread, or more
    const int threads = roles == 4 || p.page * p.D >= 4096 ? 256 : (int)(p.page * p.D / 16);
    a.q_apart = p.g_k && roles == 1 ? apart_of(p.Hq, p.Hq, p.T, p.D) : (int)p.Hq;
    const int64_t q_groups = (p.T * a.q_apart * (p.D / 16) + threads - 1) / threads;
    const int64_t groups = (int64_t)a.chunks * ((2 * p.Hkv + roles - 1) / roles) + q_groups;
    const size_t lds = (size_t)p.page * p.D * 2 + 16;
    auto kernel = a.g_k ? (roles == 4 ? kv_append_kernel<4, true> : kv_append_kernel<1, true>)
                        : (roles == 4 ? kv_append_kernel<4, false> : kv_append_kernel<1, false>);
    kernel<<<dim3((unsigned)groups), threads, lds, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

int agq_launch_qk_norm_rope(const AgqQkNormRope &p, void *stream) {
    HeadsArgs a;
    a.q = (const uint16_t *)p.q, a.k = (const uint16_t *)p.k, a.g_q = (const uint16_t *)p.g_q, a.g_k = (const uint16_t *)p.g_k;
    a.q_out = (uint16_t *)p.q_out, a.k_out = (uint16_t *)p.k_out;
    a.ldq = p.ldq, a.ldk = p.ldk, a.ldgq = p.ldgq, a.ldgk = p.ldgk, a.ldqo = p.ldqo, a.ldko = p.ldko;
    a.pos = p.pos, a.cos_t = p.rope_cos, a.sin_t = p.rope_sin, a.eps = p.eps;
    a.T = (int)p.T, a.Hq = (int)p.Hq, a.Hkv = (int)p.Hkv, a.D = (int)p.D, a.per_log2 = log2_of(p.D) - 4, a.P = (int)p.P;
    a.q_apart = apart_of(p.Hq, p.Hq + p.Hkv, p.T, p.D), a.k_apart = apart_of(p.Hkv, p.Hq + p.Hkv, p.T, p.D);
    const dim3 grid((unsigned)((p.T * (a.q_apart + a.k_apart) * (p.D / 16) + 255) / 256));
    if (p.rope_cos)
        qk_norm_rope_kernel<true><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    else
        qk_norm_rope_kernel<false><<<grid, 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}
