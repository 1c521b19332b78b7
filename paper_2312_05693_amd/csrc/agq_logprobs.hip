// Log probabilities of given tokens, entropy and the likeliest tokens of rows of logits.
#include "agq_device.h"
#include "agq_internal.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();

struct Args {
    const void *logits;
    int64_t V, ld;
    float scale;
    int n_top;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_idx;
};
template <class E>
__device__ __forceinline__ float value(E x) { return (float)x; }

// A workgroup to a row.  With c = scale log2(e) and m = max(x): z = (x - m) c, S = sum 2^z, E = sum z 2^z, log p =
// (z - log2 S) ln 2 and the entropy (log2 S - E / S) ln 2.  (x c - m c by one multiply-add would be off by m c's rounding,
// which is more than an exponent can take where the logits times scale are large.)  Alternatives: n_top passes, each for the
// best one behind the one before.
template <class E>
__global__ __launch_bounds__(256) void logprobs_kernel(const Args a) {
    __shared__ float f[3][4];
    __shared__ int who[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t = blockIdx.x;
    const E *x = (const E *)a.logits + t * a.ld;
    const int V = (int)a.V;
    const float c = a.scale * kLog2e;
    float top = -kInf;
    bool nan = false;
    for (int v = tid; v < V; v += 256) {
        const float y = value(x[v]);
        nan |= y != y;
        top = fmaxf(top, y);
    }
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) f[0][wave] = top;
    nan = __syncthreads_or(nan);
    top = fmaxf(fmaxf(f[0][0], f[0][1]), fmaxf(f[0][2], f[0][3]));
    const bool none = nan || top == kInf || top == -kInf;      // no distribution
    float S = 0.0f, H = 0.0f;
    if (!none)
        for (int v = tid; v < V; v += 256) {
            const float z = (value(x[v]) - top) * c, e = __builtin_amdgcn_exp2f(z);
            S += e;
            H += e > 0.0f ? e * z : 0.0f;
        }
    for (int m = 1; m < 64; m <<= 1) S += __shfl_xor(S, m), H += __shfl_xor(H, m);
    if (lane == 0) f[1][wave] = S, f[2][wave] = H;
    __syncthreads();
    S = (f[1][0] + f[1][1]) + (f[1][2] + f[1][3]), H = (f[2][0] + f[2][1]) + (f[2][2] + f[2][3]);
    const float lse = none ? __builtin_nanf("") : (float)log2((double)S);      // the instruction's log2(1) is -5e-8
    if (tid == 0 && a.logprob) {
        const int v = a.tokens[t];
        a.logprob[t] = (unsigned)v < (unsigned)V && !none ? ((value(x[v]) - top) * c - lse) * kLn2 : __builtin_nanf("");
    }
    if (tid == 0 && a.entropy) a.entropy[t] = (lse - H / S) * kLn2;
    float last = kInf;
    int last_at = -1;
    for (int n = 0; n < a.n_top; ++n) {
        float best = -kInf;
        int at = V;
        if (!none)
            for (int v = tid; v < V; v += 256) {
                const float y = value(x[v]);
                if ((y < last || (y == last && v > last_at)) && (at == V || y > best)) best = y, at = v;
            }
        for (int m = 1; m < 64; m <<= 1) {
            const float y = __shfl_xor(best, m);
            const int v = __shfl_xor(at, m);
            if (v < V && (at == V || y > best || (y == best && v < at))) best = y, at = v;
        }
        __syncthreads();
        if (lane == 0) f[0][wave] = best, who[wave] = at;
        __syncthreads();
        for (int w = 0; w < 4; ++w)
            if (who[w] < V && (at == V || f[0][w] > best || (f[0][w] == best && who[w] < at))) best = f[0][w], at = who[w];
        if (tid == 0) {
            a.top_idx[t * a.n_top + n] = none ? -1 : at;
            a.top_logprob[t * a.n_top + n] = none ? lse : ((best - top) * c - lse) * kLn2;
        }
        last = best, last_at = at;
    }
}

}  // namespace

int agq_launch_logprobs(const AgqLogprobs &p, void *workspace, void *stream) {
    (void)workspace;
    const Args a = {p.logits, p.V, p.ld, p.scale, (int)p.n_top, p.tokens, p.logprob, p.entropy, p.top_logprob, p.top_idx};
    if (p.kind == 1)
        logprobs_kernel<float><<<dim3((unsigned)p.T), 256, 0, (hipStream_t)stream>>>(a);
    else
        logprobs_kernel<_Float16><<<dim3((unsigned)p.T), 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}
