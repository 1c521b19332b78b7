// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
//
// One pass over the logits.  With c = scale log2(e) and m a logit near the largest so far: z = (x - m) c, S = sum 2^z, E = sum z 2^z, in
// every lane by itself and brought to a larger m when one comes that is more than 1 / c above.  (x c - m c by one multiply-add would
// be off by m c's rounding, which is more than an exponent can take where the logits times scale are large.)  Then
// log p = (x - m) scale - ln S and the entropy ln S - E / S (scale / c), of the row's joined sums in float64.
// Sums in float32 are those of the values of a load and of a unit's four loads; units are added in float64, as sums of nearly equal
// terms are off the same way at every step (rows of 131072 logits, a few larger than the others: log probabilities off by 4.6e-6,
// 4.4e-7 like this).  m stays where a larger logit is less than a factor of two above it, so that there are no more factors
// 2^(old m - new m), each rounded, than powers of two between a logit and the largest.  With d = 2^-24 S is off, relatively and to first order, by
//   4 d |difference| of z (a subtraction, a product, c's two roundings), 2 d of 2^z, 10 d of the chains, 2 d and 3 d |difference| of the
//   factors, and 10 d of the joins of lanes, wavefronts and pieces, a factor each.
// (300 rows of 128000 fp16 logits 19.8 -> 20.6 us against float32 throughout, other sizes 0 to 2 %.  A chain for each load side by
// side took registers: 4096 rows of 32000 with 20 alternatives 77 us, 74.5 with the loads one after the other.)
// The pass also leaves the largest logit of every group of neighbours (256 bytes of them: sixteen lanes' loads).  The n_top
// likeliest tokens lie in the n_top groups with the largest of these, equal ones by their place: any other token has one at
// least as good in front of it in each of those.  So only some groups are looked at again.
//
// Bound and time (replayed graph):
//   many rows by memory and the exponentials beside it: 4096 rows of 32000, fp16, 51 us: 262 MB at 5.1 TB/s, where a read alone
//     reaches 6.05; a lane's 128 logits and its share of the joins take nine instructions a logit, one of them a quarter-rate
//     exponential, 40 us of arithmetic beside it;
//   few rows by latency: 1 x 32000 with 20 alternatives 10.8 us, 64 x 128000 15.6, 200 x 50000 of float32 with a mask 16.2, of which
//     the alternatives are 4 to 5 us: the groups' order, the loads of the best ones, the order of their tokens, one after the other.
#include <limits.h>
#include "agq_device.h"
#include "agq_internal.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();
constexpr int kLoads = AGQ_LP_LOADS;       // 16-byte loads of a lane in a unit

struct Args {
    const void *logits;
    int64_t ld;
    int V, n_top, units, wave_units, pieces, groups;     // units of a row, of a wavefront; workgroups, groups of a row
    float scale;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_idx;
    struct Part *parts;          // [T][pieces]
    int32_t *tops;               // [T][groups]
};
struct Part {
    double S, E;
    float m;
    int pad;
};

// order-preserving: a < b as numbers <=> order(a) < order(b) as ints; both zeros are one, NaN does not matter
__device__ __forceinline__ int order(float x) {
    const int u = __float_as_int(x + 0.0f);
    return u ^ ((u >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float number(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7FFFFFFF)); }
// a token's place in the row's order as one number: larger logits first, then lower tokens
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(int ordered, uint32_t at) { return (Key)((uint32_t)ordered ^ 0x80000000u) << 32 | (uint32_t)~at; }

template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false); }
__device__ __forceinline__ int row_max(int v) {          // of sixteen lanes
    v = max(v, dpp<0x121>(v));                            // row_ror 1, 2, 4, 8
    v = max(v, dpp<0x122>(v));
    v = max(v, dpp<0x124>(v));
    return max(v, dpp<0x128>(v));
}

// One 16-byte load, its values less m, and the largest of them
template <class E>
struct Vec;
template <>
struct Vec<_Float16> {
    static constexpr int N = 8;
    uint32_t w[4];
    // a half of a word as float32, plus -m: one instruction
    __device__ __forceinline__ float less(int k, float minus_m) const {
        float d;
        if (k & 1)
            asm("v_fma_mix_f32 %0, %1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(w[k >> 1]), "v"(minus_m));
        else
            asm("v_fma_mix_f32 %0, %1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(w[k >> 1]), "v"(minus_m));
        return d;
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t x, uint32_t y) {      // of two pairs
        uint32_t r;
        asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
        return r;
    }
    __device__ __forceinline__ float largest() const {
        const agq_h2v h = __builtin_bit_cast(agq_h2v, max2(max2(w[0], w[1]), max2(w[2], w[3])));
        return fmaxf((float)h[0], (float)h[1]);
    }
    __device__ __forceinline__ void set(int k, _Float16 x) {
        const uint32_t u = __builtin_bit_cast(uint16_t, x);
        w[k >> 1] = k & 1 ? (w[k >> 1] & 0xFFFFu) | u << 16 : u;
    }
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    float v[4];
    __device__ __forceinline__ float less(int k, float minus_m) const { return v[k] + minus_m; }
    __device__ __forceinline__ float largest() const { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }
    __device__ __forceinline__ void set(int k, float x) { v[k] = x; }
};
template <class E>
struct Unit {
    Vec<E> d[kLoads];
};

// A lane's loads of unit u: load i holds values from (u kLoads + i) 64 N + lane N on; -infinity behind the row's end.  The rows
// begin at any element: the loads need not be aligned.  (Loads that leave nothing in the caches are faster where the logits come from
// memory, 4096 x 32000 51.0 -> 48.3 us, and slower behind the product that has just made them, 500 x 128000 31.1 -> 33.7.)
template <class E>
__device__ __forceinline__ Unit<E> load_unit(const E *x, int V, int u, int lane) {
    constexpr int N = Vec<E>::N;
    Unit<E> r;
    const int64_t at = (int64_t)u * kLoads * 64 * N + lane * N;
    if ((int64_t)(u + 1) * kLoads * 64 * N <= V) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) __builtin_memcpy(&r.d[i], x + at + i * 64 * N, 16);
        return r;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int64_t e = at + i * 64 * N;
        if (e + N <= V) {
            __builtin_memcpy(&r.d[i], x + e, 16);
            continue;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) r.d[i].set(k, e + k < V ? x[e + k] : (E)-kInf);
    }
    return r;
}

struct Sums {
    double S, E;
    float m;
};
// The sums of a unit's values relative to m, a chain for each load.  Where 2^z is 0 its product with z is to be 0 too, also for
// z = -infinity: CLAMP keeps z finite there.
template <class E, bool CLAMP>
__device__ __forceinline__ void sum_values(float &S, float &H, const Unit<E> &u, float m, float c) {
    S = 0.0f, H = 0.0f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        float s, h;
#pragma unroll
        for (int k = 0; k < Vec<E>::N; ++k) {
            const float z = u.d[i].less(k, -m) * c, e = __builtin_amdgcn_exp2f(z), y = CLAMP ? fmaxf(z, -150.0f) : z;
            s = k ? s + e : e;
            h = k ? fmaf(e, y, h) : e * y;
        }
        S = i ? S + s : s, H = i ? H + h : h;
    }
}
// a lane's sums taken to a larger m, and a unit's values into them
template <class E, bool TOP>
__device__ __forceinline__ void add_unit(Sums &s, const Unit<E> &u, float c, int *tops, int lane) {
    float top[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) top[i] = u.d[i].largest();
    const float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    if constexpr (TOP) {                                  // lane i of sixteen writes load i's
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int o = row_max(order(top[i]));
            mine = (lane & 15) == i ? o : mine;
        }
        if ((lane & 15) < kLoads) tops[(lane & 15) * 4 + (lane >> 4)] = mine;
    }
    const bool past = (all - s.m) * c > 1.0f;             // always where s.m is not a logit yet
    if (__any(past)) {
        const float m = past ? all : s.m, d = fmaxf((s.m - m) * c, -150.0f);
        const double f = (double)__builtin_amdgcn_exp2f(d);
        s.E = f * fma((double)d, s.S, s.E), s.S *= f, s.m = m;
    }
    float S, H;
    sum_values<E, false>(S, H, u, s.m, c);
    if (__any(H != H)) sum_values<E, true>(S, H, u, s.m, c);     // -infinity among them, or a NaN (which stays one)
    s.S += (double)S, s.E += (double)H;
}

struct Row {
    double S, E;
    float m;
};
__device__ __forceinline__ Row taken_to(const Row &r, float m, float c) {
    const float d = fmaxf((r.m - m) * c, -300.0f);
    const double f = (double)__builtin_amdgcn_exp2f(d);
    return Row{f * r.S, f * (r.E + (double)d * r.S), m};
}
__device__ __forceinline__ Row joined(const Row &a, const Row &b, float c) {
    const float m = fmaxf(a.m, b.m);
    const Row x = taken_to(a, m, c), y = taken_to(b, m, c);
    return Row{x.S + y.S, x.E + y.E, m};
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double v) {     // plus another lane's, in the rows that are written; 0 elsewhere
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
    return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {    // in lane 63
    v = dpp_add<0x111, 0xF>(v);                           // row_shr 1, 2, 4, 8: inside sixteen lanes
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);                           // row_bcast 15 and 31
    return dpp_add<0x143, 0xC>(v);
}
// the wavefront's rows joined; S and E in lane 63 only
__device__ __forceinline__ Row wave_joined(Row r, float c) {
    float m = r.m;
    m = fmaxf(m, __int_as_float(dpp<0x121>(__float_as_int(m))));
    m = fmaxf(m, __int_as_float(dpp<0x122>(__float_as_int(m))));
    m = fmaxf(m, __int_as_float(dpp<0x124>(__float_as_int(m))));
    m = fmaxf(m, __int_as_float(dpp<0x128>(__float_as_int(m))));
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    r = taken_to(r, m, c);
    return Row{wave_sum(r.S), wave_sum(r.E), m};
}
__device__ __forceinline__ double lane_63(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)u, 63));
}

// ---------------------------------------------------------------- the likeliest tokens, by four wavefronts
constexpr int kBlock = 16;       // groups' largest logits that a lane holds at once
constexpr int kAtOnce = 4;       // groups that a wavefront looks at together
constexpr int kWaiting = 64 + 128 * kAtOnce;
struct Scratch {
    Key waiting[4 * kWaiting];   // of tokens that are not in a list yet, a quarter to each wavefront; before that of groups
    Key best[4][64];             // the wavefronts' lists
    int group[64], picked;       // groups to be looked at
    Key cut;
};

// the key of lane ^ X, by data-parallel moves
template <int X>
__device__ __forceinline__ uint32_t other(uint32_t v, int lane) {
    if constexpr (X == 1) return (uint32_t)dpp<0xB1>((int)v);             // quad_perm 1 0 3 2
    if constexpr (X == 2) return (uint32_t)dpp<0x4E>((int)v);             // quad_perm 2 3 0 1
    if constexpr (X == 4) {                                               // row_ror 4 and 12: four lanes back, four ahead
        const int back = dpp<0x124>((int)v), ahead = dpp<0x12C>((int)v);
        return (uint32_t)(lane & 4 ? back : ahead);
    }
    if constexpr (X == 8) return (uint32_t)dpp<0x128>((int)v);            // row_ror 8
    if constexpr (X == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return lane & 16 ? r[0] : r[1];
    }
    if constexpr (X == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return lane & 32 ? r[0] : r[1];
    }
}
template <int X>
__device__ __forceinline__ Key other(Key k, int lane) { return (Key)other<X>((uint32_t)(k >> 32), lane) << 32 | other<X>((uint32_t)k, lane); }
__device__ __forceinline__ Key better(Key a, Key b) { return a > b ? a : b; }
// a step of a sorting network: the better one of lanes X apart to the lower one if `down`, else to the upper one
template <int X>
__device__ __forceinline__ Key step(Key k, int lane, bool down) {
    const Key o = other<X>(k, lane);
    return (k > o) == (((lane & X) == 0) == down) ? k : o;
}
template <int X>
__device__ __forceinline__ Key steps(Key k, int lane, bool down) {
    k = step<X>(k, lane, down);
    if constexpr (X > 1) k = steps<X / 2>(k, lane, down);
    return k;
}
// the wavefront's keys in ascending order
__device__ __forceinline__ Key sorted(Key k, int lane) {
    k = steps<1>(k, lane, (lane & 2) != 0);
    k = steps<2>(k, lane, (lane & 4) != 0);
    k = steps<4>(k, lane, (lane & 8) != 0);
    k = steps<8>(k, lane, (lane & 16) != 0);
    k = steps<16>(k, lane, (lane & 32) != 0);
    return steps<32>(k, lane, false);
}
// the best 64 of a descending and an ascending list, descending
__device__ __forceinline__ Key merged(Key a, Key b, int lane) { return steps<32>(better(a, b), lane, true); }
__device__ __forceinline__ Key lane_key(Key k, int lane) {
    return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// The best n of the keys that come by: those that wait (in LDS) are merged into `list` (descending, lane i has the i-th), 64 at a
// time, once there are 64 or with ALL; cut: the n-th, below which none counts.
struct Best {
    Key list, cut;
    int waiting, n, lane;
    Key *wait;
    __device__ __forceinline__ void fence() const { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
    __device__ __forceinline__ void add(Key k, bool good) {
        const unsigned long long in = __ballot(good);
        if (good) wait[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = k;
        waiting += __popcll(in);
    }
    __device__ __forceinline__ void merge(bool all) {
        fence();
        int q = 0;
#pragma unroll 1
        for (; q + 64 <= waiting || (all && q < waiting); q += 64) {
            const Key k = q + lane < waiting ? wait[q + lane] : 0;
            if (!__any(k > cut)) continue;
            list = merged(list, sorted(k, lane), lane);
            const Key last = lane_key(list, n - 1);
            if (last != 0) cut = last;
        }
        if (q == 0) return;
        const Key k = q + lane < waiting ? wait[q + lane] : 0;
        fence();
        wait[lane] = k;
        fence();
        waiting = max(waiting - q, 0);
    }
};

// The first wavefront finds the groups.
template <class E>
__device__ __forceinline__ void find_groups(const int *tops, int groups, int n, Scratch &sc, int lane) {
    // every lane's best group; the n-th best of these lets the n best groups and few others through
    int top[kBlock];
    auto load_tops = [&](int g0) {
#pragma unroll
        for (int i = 0; i < kBlock; ++i) top[i] = tops[min(g0 + 64 * i + lane, groups - 1)];
#pragma unroll
        for (int i = 0; i < kBlock; ++i) top[i] = g0 + 64 * i + lane < groups ? top[i] : INT_MIN;
    };
    Key mine = 0;
#pragma unroll 1
    for (int g0 = 0; g0 < groups; g0 += 64 * kBlock) {
        load_tops(g0);
        int best = top[0], at = g0;
#pragma unroll
        for (int i = 1; i < kBlock; ++i) {
            at = top[i] > best ? g0 + 64 * i : at;
            best = max(best, top[i]);
        }
        if (best != INT_MIN) mine = better(mine, key_of(best, (uint32_t)(at + lane)));
    }
    // The n best groups, a lane each (all of them if there are no more).  Where few were let through, these will do.
    const Key bound = n <= min(groups, 64) ? lane_key(sorted(mine, lane), 64 - n) : 0;
    Best g = {0, bound ? bound - 1 : 0, 0, n, lane, sc.waiting};
#pragma unroll 1
    for (int g0 = 0; g0 < groups; g0 += 64 * kBlock) {
        if (groups > 64 * kBlock) load_tops(g0);
#pragma unroll
        for (int i = 0; i < kBlock; ++i) {
            if (g0 + 64 * i >= groups) break;
            const Key k = key_of(top[i], (uint32_t)(g0 + 64 * i + lane));
            g.add(k, top[i] != INT_MIN && k > g.cut);
        }
        if (g.waiting > 64 || groups > 64 * kBlock) g.merge(g0 + 64 * kBlock >= groups);
    }
    g.fence();
    int picked = g.waiting;
    Key least = bound;
    if (picked > 0) {
        g.list = lane < picked ? g.wait[lane] : 0;
    } else {
        picked = n;
        least = lane_key(g.list, n - 1);
    }
    sc.group[lane] = (int)~(uint32_t)g.list;
    if (lane == 0) sc.picked = picked, sc.cut = least & ~(Key)0xFFFFFFFFu;       // tokens as large as the n-th group's largest
}

// Each of four wavefronts looks at a quarter of them; the first one joins what they found.  Lane i < n of it gets the i-th best
// token's key.  Called by the whole workgroup, behind a barrier.
template <class E>
__device__ __forceinline__ Key likeliest(const E *x, int V, int n, Scratch &sc, int wave, int lane) {
    constexpr int G = 16 * Vec<E>::N, PER = G / 64;
    static_assert(4 * kWaiting >= 64 + 64 * kBlock, "a block of groups may wait");
    if (wave < 4) {
        const int picked = sc.picked;
        Best b = {0, sc.cut, 0, n, lane, sc.waiting + wave * kWaiting};
#pragma unroll 1
        for (int p0 = wave; p0 < picked; p0 += 4 * kAtOnce) {
            E v[kAtOnce][PER];
            int at[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                at[i] = p0 + 4 * i < picked ? __builtin_amdgcn_readfirstlane(sc.group[p0 + 4 * i]) * G + lane : V;
#pragma unroll
                for (int k = 0; k < PER; ++k) v[i][k] = x[min(at[i] + 64 * k, V - 1)];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const Key key = key_of(order((float)v[i][k]), (uint32_t)(at[i] + 64 * k));
                    b.add(key, at[i] + 64 * k < V && key > b.cut);
                }
            b.merge(p0 + 4 * kAtOnce >= picked);
        }
        sc.best[wave][lane] = b.list;
    }
    __syncthreads();
    Key list = 0;
    if (wave == 0) {
        list = sc.best[0][lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) list = merged(list, sc.best[w][63 - lane], lane);
    }
    return list;
}

// What is asked for of a row, by a workgroup.  r and tops are the first wavefront's.
template <class E, bool TOP>
__device__ __forceinline__ void answer(const Args &a, int64_t t, const E *x, const Row &r, const int *tops, Scratch &sc, int wave, int lane) {
    const double scale = (double)a.scale;
    double lse = 0.0;
    if (wave == 0) {
        const bool none = !(r.S > 0.0);    // no distribution: a NaN, or +infinity (less itself), made it one; -infinity only, 0
        lse = none ? __builtin_nan("") : log(r.S);
        if (lane == 0) {
            if (a.logprob) {
                const int v = a.tokens[t];
                a.logprob[t] = (float)((unsigned)v < (unsigned)a.V ? ((double)(float)x[v] - (double)r.m) * scale - lse : __builtin_nan(""));
            }
            if (a.entropy) a.entropy[t] = (float)(lse - r.E / r.S * (scale / (double)(a.scale * kLog2e)));
        }
        if constexpr (TOP) {
            if (none) {
                if (lane == 0) sc.picked = 0;
            } else {
                find_groups<E>(tops, a.groups, a.n_top, sc, lane);
            }
        }
    }
    if constexpr (TOP) {
        __syncthreads();
        const Key k = likeliest<E>(x, a.V, a.n_top, sc, wave, lane);
        if (wave == 0 && lane < a.n_top) {
            const bool none = lse != lse;
            a.top_idx[t * a.n_top + lane] = none ? -1 : (int)~(uint32_t)k;
            a.top_logprob[t * a.n_top + lane] = (float)(((double)number((int)((uint32_t)(k >> 32) ^ 0x80000000u)) - (double)r.m) * scale - lse);
        }
    }
}

// A workgroup to a piece of a row: wave_units units of each of its wavefronts, the next one on its way while one is added up.  WHOLE: the piece is the row, and the answers
// follow here.
template <class E, bool TOP, bool WHOLE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void logprobs_kernel(const Args a) {
    __shared__ Row rows[WAVES];
    __shared__ int held[WHOLE && TOP ? AGQ_LP_HELD : 1];
    __shared__ Scratch sc;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int piece = WHOLE ? 0 : blockIdx.x % a.pieces;
    const int64_t t = WHOLE ? blockIdx.x : blockIdx.x / a.pieces;
    const E *x = (const E *)a.logits + t * a.ld;
    const float c = a.scale * kLog2e;
    int *tops = WHOLE ? held : a.tops + t * a.groups;
    Sums s = {0.0, 0.0, -3.402823466e38f};
    const int u0 = (piece * WAVES + wave) * a.wave_units, u1 = min(u0 + a.wave_units, a.units);
    if (u0 < u1) {
        Unit<E> next = load_unit(x, a.V, u0, lane);
        for (int u = u0; u < u1; ++u) {
            const Unit<E> now = next;
            if (u + 1 < u1) next = load_unit(x, a.V, u + 1, lane);
            add_unit<E, TOP>(s, now, c, tops + u * kLoads * 4, lane);
        }
    }
    Row r = wave_joined(Row{s.S, s.E, s.m}, c);
    if constexpr (WAVES > 1) {
        if (lane == 63) rows[wave] = r;
        __syncthreads();
    }
    if (wave > 0) {
        if constexpr (!(WHOLE && TOP)) return;
    } else if constexpr (WAVES == 1) {
        r.S = lane_63(r.S), r.E = lane_63(r.E);
    } else if constexpr (WAVES == 2) {
        r = joined(rows[0], rows[1], c);
    } else if constexpr (WAVES == 4) {
        r = joined(joined(rows[0], rows[1], c), joined(rows[2], rows[3], c), c);
    } else {
        r = wave_joined(lane < WAVES ? rows[lane] : Row{0.0, 0.0, -3.402823466e38f}, c);
        r.S = lane_63(r.S), r.E = lane_63(r.E);
    }
    if constexpr (WHOLE) {
        answer<E, TOP>(a, t, x, r, tops, sc, wave, lane);
    } else if (lane == 0) {
        a.parts[t * a.pieces + piece] = Part{r.S, r.E, r.m, 0};
    }
}

// the answers of rows whose pieces were several workgroups'
template <class E, bool TOP>
__global__ __launch_bounds__(TOP ? 256 : 64) void join_kernel(const Args a) {
    __shared__ Scratch sc;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x;
    const float c = a.scale * kLog2e;
    Row r = {0.0, 0.0, -3.402823466e38f};
    if (wave == 0) {
        const Part *parts = a.parts + t * a.pieces;
        Part q = {0.0, 0.0, -3.402823466e38f, 0};
        if (lane < a.pieces) q = parts[lane];
        float m = q.m;
        for (int p = lane + 64; p < a.pieces; p += 64) m = fmaxf(m, parts[p].m);      // one factor to each piece
        r = taken_to(Row{q.S, q.E, q.m}, m, c);
        for (int p = lane + 64; p < a.pieces; p += 64) {
            const Part o = parts[p];
            const Row x = taken_to(Row{o.S, o.E, o.m}, m, c);
            r.S += x.S, r.E += x.E;
        }
        r = wave_joined(r, c);
        r.S = lane_63(r.S), r.E = lane_63(r.E);
    }
    answer<E, TOP>(a, t, (const E *)a.logits + t * a.ld, r, a.tops + t * a.groups, sc, wave, lane);
}

template <class E, bool TOP>
int launch(const Args &a, int64_t T, const AgqLpPlan &p, hipStream_t st) {
    const dim3 grid((unsigned)(T * p.pieces));
    if (p.whole) {
        auto kernel = p.waves == 16 ? logprobs_kernel<E, TOP, true, 16> : logprobs_kernel<E, TOP, true, 4>;
        if constexpr (!TOP) kernel = p.waves == 1 ? logprobs_kernel<E, false, true, 1> : p.waves == 2 ? logprobs_kernel<E, false, true, 2> : kernel;
        kernel<<<grid, 64 * p.waves, 0, st>>>(a);
        return (int)hipGetLastError();
    }
    logprobs_kernel<E, TOP, false, 4><<<grid, 256, 0, st>>>(a);
    if (int err = (int)hipGetLastError()) return err;
    join_kernel<E, TOP><<<dim3((unsigned)T), TOP ? 256 : 64, 0, st>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

size_t agq_logprobs_workspace(int64_t T, int64_t V, int kind, int64_t n_top) {
    const AgqLpPlan p = agq_lp_plan(T, V, kind, n_top);
    return p.whole ? 0 : (size_t)T * ((size_t)p.pieces * sizeof(Part) + (n_top ? (size_t)p.groups * 4 : 0));
}

int agq_launch_logprobs(const AgqLogprobs &p, void *workspace, void *stream) {
    const AgqLpPlan plan = agq_lp_plan(p.T, p.V, p.kind, p.n_top);
    Part *parts = (Part *)workspace;
    const Args a = {p.logits, p.ld, (int)p.V, (int)p.n_top, plan.units, plan.wave_units, plan.pieces, plan.groups, p.scale, p.tokens, p.logprob, p.entropy,
                    p.top_logprob, p.top_idx, parts, plan.whole ? nullptr : (int32_t *)(parts + p.T * plan.pieces)};
    hipStream_t st = (hipStream_t)stream;
    if (p.kind) return p.n_top ? launch<float, true>(a, p.T, plan, st) : launch<float, false>(a, p.T, plan, st);
    return p.n_top ? launch<_Float16, true>(a, p.T, plan, st) : launch<_Float16, false>(a, p.T, plan, st);
}
