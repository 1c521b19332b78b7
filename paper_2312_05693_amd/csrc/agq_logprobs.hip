// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
//
// One pass over the logits.  With c = scale log2(e) and m the largest logit so far: z = (x - m) c, S = sum 2^z, E = sum z 2^z, in
// every lane by itself and brought to a larger m when one comes.  (x c - m c by one multiply-add would be off by m c's
// rounding, which is more than an exponent can take where the logits times scale are large.)  Then log p = (x - m) scale - ln S
// and the entropy ln S - E / S (scale / c), of the row's joined sums in float64.
// The pass also leaves the largest logit of every group of neighbours (256 bytes of them: sixteen lanes' loads).  The n_top
// likeliest tokens lie in the n_top groups with the largest of these, equal ones by their place: any other token has one at
// least as good in front of it in each of those.  So only some groups are looked at again, by one wavefront.
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

// the values of one 16-byte load
template <class E>
struct Vec;
template <>
struct Vec<_Float16> {
    static constexpr int N = 8;
    _Float16 v[8];
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    float v[4];
};
template <class E>
struct Unit {
    Vec<E> d[kLoads];
};

// A lane's loads of unit u: load i holds values from (u kLoads + i) 64 N + lane N on; -infinity behind the row's end.  The rows
// begin at any element: the loads need not be aligned.
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
        for (int k = 0; k < N; ++k) r.d[i].v[k] = e + k < V ? x[e + k] : (E)-kInf;
    }
    return r;
}

struct Sums {
    float m, S, E;
};
// a lane's sums taken to a larger m, and a unit's values into them
template <class E, bool TOP>
__device__ __forceinline__ void add_unit(Sums &s, const Unit<E> &u, float c, int *tops, int lane) {
    constexpr int N = Vec<E>::N;
    float top[kLoads], all = s.m;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        top[i] = (float)u.d[i].v[0];
#pragma unroll
        for (int k = 1; k < N; ++k) top[i] = fmaxf(top[i], (float)u.d[i].v[k]);
        all = fmaxf(all, top[i]);
    }
    if constexpr (TOP) {                                  // lane i of sixteen writes load i's
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int o = row_max(order(top[i]));
            mine = (lane & 15) == i ? o : mine;
        }
        if ((lane & 15) < kLoads) tops[(lane & 15) * 4 + (lane >> 4)] = mine;
    }
    const float d = (s.m - all) * c, f = __builtin_amdgcn_exp2f(d);
    s.E = f * (s.E + fmaxf(d, -150.0f) * s.S);            // S is 0 where s.m is not a logit yet
    s.S *= f;
    s.m = all;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float z = ((float)u.d[i].v[k] - all) * c, e = __builtin_amdgcn_exp2f(z);
            s.S += e;
            s.E = fmaf(e, fmaxf(z, -150.0f), s.E);        // e is 0 there; -infinity times 0 would not be
        }
}

struct Row {
    double S, E;
    float m;
};
__device__ __forceinline__ Row joined(const Row &a, const Row &b, float c) {
    Row r;
    r.m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - r.m) * c, -300.0f), db = fmaxf((b.m - r.m) * c, -300.0f);
    const double fa = (double)__builtin_amdgcn_exp2f(da), fb = (double)__builtin_amdgcn_exp2f(db);
    r.S = a.S * fa + b.S * fb;
    r.E = fa * (a.E + (double)da * a.S) + fb * (b.E + (double)db * b.S);
    return r;
}
__device__ __forceinline__ Row wave_joined(Row r, float c) {
    for (int s = 1; s < 64; s <<= 1) r = joined(r, Row{__shfl_xor(r.S, s), __shfl_xor(r.E, s), __shfl_xor(r.m, s)}, c);
    return r;
}

// ---------------------------------------------------------------- the likeliest tokens, by one wavefront
struct Scratch {
    Key waiting[128];            // candidates that are not in the list yet
    int picked[256];             // groups to be looked at
};

__device__ __forceinline__ Key other(Key k, int x) { return (Key)__shfl_xor((long long)k, x); }
__device__ __forceinline__ Key better(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key worse(Key a, Key b) { return a > b ? b : a; }
// the wavefront's keys in descending order
__device__ __forceinline__ Key sorted(Key k, int lane) {
#pragma unroll
    for (int n = 2; n <= 64; n <<= 1)
#pragma unroll
        for (int j = n >> 1; j > 0; j >>= 1) {
            const Key o = other(k, j);
            k = (((lane & n) == 0) == ((lane & j) == 0)) ? better(k, o) : worse(k, o);
        }
    return k;
}
// the best 64 of two descending lists, descending
__device__ __forceinline__ Key merged(Key a, Key b, int lane) {
    Key k = better(a, (Key)__shfl((long long)b, 63 - lane));
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) {
        const Key o = other(k, j);
        k = (lane & j) == 0 ? better(k, o) : worse(k, o);
    }
    return k;
}
__device__ __forceinline__ Key lane_key(Key k, int lane) {
    return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// lane i < n gets the i-th best token's key
template <class E>
__device__ __forceinline__ Key likeliest(const E *x, int V, const int *tops, int groups, int n, Scratch &sc, int lane) {
    constexpr int G = 16 * Vec<E>::N, PER = G / 64;
    // each lane's best group; the n-th best of these lets the n best groups and few others through
    Key mine = 0;
    for (int g = lane; g < groups; g += 64) mine = better(mine, key_of(tops[g], (uint32_t)g));
    Key bound = 0;
    if (n <= min(groups, 64)) {
        int before = 0;
        for (int l = 0; l < 64; ++l) before += lane_key(mine, l) > mine;
        bound = lane_key(mine, __ffsll((long long)__ballot(before == n - 1)) - 1);
    }
    Key list = 0, cut = bound & ~(Key)0xFFFFFFFFu;       // tokens above it: at first those as large as the bound's
    int picked = 0, waiting = 0;
    auto take = [&] {                                     // the first 64 that wait, into the list
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const Key k = lane < waiting ? sc.waiting[lane] : 0, rest = lane + 64 < waiting ? sc.waiting[lane + 64] : 0;
        list = merged(list, sorted(k, lane), lane);
        sc.waiting[lane] = rest;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        waiting = max(waiting - 64, 0);
        const Key last = lane_key(list, n - 1);
        if (last != 0) cut = last;
    };
    auto look = [&] {
        constexpr int AT_ONCE = 8;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int p0 = 0; p0 < picked; p0 += AT_ONCE) {
            E v[AT_ONCE][PER];
            int at[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                at[i] = p0 + i < picked ? sc.picked[p0 + i] * G + lane : V;
#pragma unroll
                for (int k = 0; k < PER; ++k) v[i][k] = at[i] + 64 * k < V ? x[at[i] + 64 * k] : (E)0;
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const int a = at[i] + 64 * k;
                    const Key key = a < V ? key_of(order((float)v[i][k]), (uint32_t)a) : 0;
                    const unsigned long long in = __ballot(key > cut);
                    if (in == 0) continue;
                    if (key > cut) sc.waiting[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = key;
                    waiting += __popcll(in);
                    if (waiting >= 64) take();
                }
        }
        picked = 0;
    };
    for (int g0 = 0; g0 < groups; g0 += 64) {
        const int g = g0 + lane;
        const bool pick = g < groups && key_of(tops[g], (uint32_t)g) >= bound;
        const unsigned long long in = __ballot(pick);
        if (pick) sc.picked[picked + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = g;
        picked += __popcll(in);
        if (picked > 192) look();
    }
    look();
    if (waiting > 0) take();
    return list;
}

// what is asked for of a row, by one wavefront
template <class E>
__device__ __forceinline__ void answer(const Args &a, int64_t t, const E *x, const Row &r, const int *tops, Scratch &sc, int lane) {
    const bool none = !(r.S > 0.0);        // no distribution: a NaN, or +infinity (less itself), made it one; -infinity only, 0
    const double nan = __builtin_nan(""), lse = none ? nan : log(r.S), scale = (double)a.scale;
    if (lane == 0) {
        if (a.logprob) {
            const int v = a.tokens[t];
            a.logprob[t] = (float)((unsigned)v < (unsigned)a.V ? ((double)(float)x[v] - (double)r.m) * scale - lse : nan);
        }
        if (a.entropy) a.entropy[t] = (float)(lse - r.E / r.S * (scale / (double)(a.scale * kLog2e)));
    }
    if (a.n_top == 0) return;
    const Key k = none ? 0 : likeliest<E>(x, a.V, tops, a.groups, a.n_top, sc, lane);
    if (lane < a.n_top) {
        a.top_idx[t * a.n_top + lane] = none ? -1 : (int)~(uint32_t)k;
        a.top_logprob[t * a.n_top + lane] = (float)(((double)number((int)((uint32_t)(k >> 32) ^ 0x80000000u)) - (double)r.m) * scale - lse);
    }
}

// A workgroup to a piece of a row: wave_units units of each of its four wavefronts.  WHOLE: the piece is the row, and the
// answers follow here.
template <class E, bool TOP, bool WHOLE>
__global__ __launch_bounds__(256) void logprobs_kernel(const Args a) {
    __shared__ Row rows[4];
    __shared__ int held[WHOLE && TOP ? AGQ_LP_HELD : 1];
    __shared__ Scratch sc;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int piece = WHOLE ? 0 : blockIdx.x % a.pieces;
    const int64_t t = WHOLE ? blockIdx.x : blockIdx.x / a.pieces;
    const E *x = (const E *)a.logits + t * a.ld;
    const float c = a.scale * kLog2e;
    int *tops = WHOLE ? held : a.tops + t * a.groups;
    Sums s = {-3.402823466e38f, 0.0f, 0.0f};
    const int u0 = (piece * 4 + wave) * a.wave_units, u1 = min(u0 + a.wave_units, a.units);
    if (u0 < u1) {
        Unit<E> next = load_unit(x, a.V, u0, lane);
        for (int u = u0; u < u1; ++u) {
            const Unit<E> now = next;
            if (u + 1 < u1) next = load_unit(x, a.V, u + 1, lane);
            add_unit<E, TOP>(s, now, c, tops + u * kLoads * 4, lane);
        }
    }
    Row r = wave_joined(Row{(double)s.S, (double)s.E, s.m}, c);
    if (lane == 0) rows[wave] = r;
    __syncthreads();
    if (wave > 0) return;
    r = joined(joined(rows[0], rows[1], c), joined(rows[2], rows[3], c), c);
    if constexpr (WHOLE) {
        answer<E>(a, t, x, r, tops, sc, lane);
    } else if (lane == 0) {
        a.parts[t * a.pieces + piece] = Part{r.S, r.E, r.m, 0};
    }
}

// the answers of rows whose pieces were several workgroups'
template <class E>
__global__ __launch_bounds__(64) void join_kernel(const Args a) {
    __shared__ Scratch sc;
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x;
    const float c = a.scale * kLog2e;
    Row r = {0.0, 0.0, -3.402823466e38f};
    for (int p = lane; p < a.pieces; p += 64) {
        const Part q = a.parts[t * a.pieces + p];
        r = joined(r, Row{q.S, q.E, q.m}, c);
    }
    r = wave_joined(r, c);
    answer<E>(a, t, (const E *)a.logits + t * a.ld, r, a.tops + t * a.groups, sc, lane);
}

template <class E>
int launch(const Args &a, int64_t T, bool whole, hipStream_t st) {
    const dim3 grid((unsigned)(T * a.pieces));
    if (whole) {
        if (a.n_top)
            logprobs_kernel<E, true, true><<<grid, 256, 0, st>>>(a);
        else
            logprobs_kernel<E, false, true><<<grid, 256, 0, st>>>(a);
        return (int)hipGetLastError();
    }
    if (a.n_top)
        logprobs_kernel<E, true, false><<<grid, 256, 0, st>>>(a);
    else
        logprobs_kernel<E, false, false><<<grid, 256, 0, st>>>(a);
    if (int err = (int)hipGetLastError()) return err;
    join_kernel<E><<<dim3((unsigned)T), 64, 0, st>>>(a);
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
    return p.kind ? launch<float>(a, p.T, plan.whole, (hipStream_t)stream) : launch<_Float16>(a, p.T, plan.whole, (hipStream_t)stream);
}
