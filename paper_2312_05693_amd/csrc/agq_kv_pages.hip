// Pages of the key/value cache that several requests hold: requests that go on as copies of others, requests that lose
// tokens, pages copied and tokens moved in the caches of all layers.
#include "agq_device.h"
#include "agq_internal.h"

namespace {

constexpr int kMaxB = AGQ_KV_MAX_B;   // requests: their sums are held in LDS

// Three launches make a step: the holders' counts are copied (and listed tokens checked), every workgroup works out the
// requests' sums for itself and does its share of the rows, and the pages that nobody holds any more go to the ring.  Counts
// change by atomic additions of whole numbers, whose order does not matter; the pages given back are found afterwards in the
// order of their numbers, so the ring does not depend on it either.
// Small steps (agq_kv_one) are ONE launch of one workgroup, with the counts in LDS: all of it is waiting for memory and for launches
// (a fork of 8 requests 4.8 us, of 256 9.0, a compaction of 64 requests 6.4; three launches take 11 to 13).
template <bool ONE>
struct Sizes {
    static constexpr int THREADS = ONE ? 1024 : 512, B = ONE ? AGQ_KV_ONE_B : kMaxB, PAGES = ONE ? AGQ_KV_ONE_PAGES : 1;
};
struct Books {
    const int32_t *kv_len, *table, *shared, *free_in;
    int32_t *ring, *kv_len_out, *table_out, *shared_out, *free_out, *status;
    int32_t *copy_src, *copy_dst, *moves;       // a fork's, a compaction's; else NULL
    int64_t max_pages;
    int B, page_log2, n_pages;
};
struct ForkArgs : Books {
    const int32_t *parent;
};

__device__ __forceinline__ int ring_at(int head, int64_t i, int n_pages) {       // head and i below n_pages
    const uint32_t at = (uint32_t)head + (uint32_t)i;
    return (int)(at >= (uint32_t)n_pages ? at - (uint32_t)n_pages : at);
}

// the sum over the workgroup's threads before this one, and of all of them
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, int *waves, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int up = agq_wave_scan(v);
    __syncthreads();
    if (lane == 63) waves[wave] = up;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        total += waves[w];
    }
    return before + up - v;
}

// This workgroup's part of a table: f(request, entry).  One workgroup: thread by thread over rows and entries; else a row's
// next entries to a workgroup.
template <bool ONE, class F>
__device__ __forceinline__ void over_table(int B, int64_t max_pages, F f) {
    constexpr int THREADS = Sizes<ONE>::THREADS;
    if constexpr (ONE) {
        const unsigned most = (unsigned)max_pages, n = (unsigned)B * most;       // some thousands
        for (unsigned i = threadIdx.x; i < n; i += THREADS) f((int)(i / most), (int)(i % most));
    } else {
        const int64_t chunks = (max_pages + THREADS - 1) / THREADS;
        for (int64_t item = blockIdx.x; item < B * chunks; item += gridDim.x) f((int)(item / chunks), (int)(item % chunks) * THREADS + (int)threadIdx.x);
    }
}

// Pages whose count fell below 0 go behind the free ones, of which there were `count` from head on before the step, in the order of
// their numbers; their number.  If that is more than n_pages - count, what does not fit is not written.  The counts are written to out, 0 for those.  A thread has four neighbours of each of TILES tiles at once, whose loads are on
// their way before the first is looked at (a million pages in memory 240 us, 450 without; one tile where they are in LDS).
template <int THREADS, int TILES>
__device__ __forceinline__ int give_back(const int32_t *counts, int32_t *out, int n_pages, int32_t *ring, int head, int count) {
    constexpr int WAVES = THREADS / 64, TILE = 4 * THREADS;
    __shared__ int waves[TILES][WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t first = (uint32_t)ring_at(head, count, n_pages);
    int given = 0;
#pragma unroll 1
    for (int64_t i0 = 0; i0 < n_pages; i0 += TILES * TILE) {
        int c[TILES][4], up[TILES];
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            const int64_t i = i0 + k * TILE + threadIdx.x * 4;
            if (i + 4 <= n_pages) {
                __builtin_memcpy(c[k], counts + i, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) c[k][j] = i + j < n_pages ? counts[i + j] : 0;
            }
        }
#pragma unroll
        for (int k = 0; k < TILES; ++k) up[k] = agq_wave_scan((c[k][0] < 0) + (c[k][1] < 0) + (c[k][2] < 0) + (c[k][3] < 0));
        __syncthreads();
        if (lane == 63)
#pragma unroll
            for (int k = 0; k < TILES; ++k) waves[k][wave] = up[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            const int64_t i = i0 + k * TILE + threadIdx.x * 4;
            int at = given + up[k] - ((c[k][0] < 0) + (c[k][1] < 0) + (c[k][2] < 0) + (c[k][3] < 0));
#pragma unroll 4
            for (int w = 0; w < WAVES; ++w) {
                const int x = waves[k][w];
                at += w < wave ? x : 0;
                given += x;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c[k][j] < 0) {
                    const uint32_t r = first + (uint32_t)at;
                    if (at++ < n_pages - count) ring[r >= (uint32_t)n_pages ? r - (uint32_t)n_pages : r] = (int)i + j;
                }
                if (i + j < n_pages && (c[k][j] < 0 || out != counts)) out[i + j] = max(c[k][j], 0);
            }
        }
    }
    return given;
}

__global__ __launch_bounds__(256) void shared_copy_kernel(const int32_t *shared, int32_t *shared_out, int n_pages) {
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n_pages; i += gridDim.x * 256) shared_out[i] = max(shared[i], 0);
}

// A step that gives back more pages than were not free before it (the books contradict each other) is taken back: copies of the
// inputs, by one workgroup.  Table entries behind a request's pages and ring entries that are not free have been written by then.
template <int THREADS>
__device__ __forceinline__ void take_back(const Books &a) {
    const int tid = threadIdx.x;
    if (tid == 0) {
        *a.status = -1;
        a.free_out[0] = a.free_in[0], a.free_out[1] = a.free_in[1];
        if (a.moves) a.moves[0] = 0;
    }
    for (int i = tid; i < a.n_pages; i += THREADS) a.shared_out[i] = max(a.shared[i], 0);
    for (int b = tid; b < a.B; b += THREADS) {
        a.kv_len_out[b] = a.kv_len[b];
        if (a.copy_src) a.copy_src[b] = a.copy_dst[b] = -1;
    }
    for (int b = 0; b < a.B; ++b) {
        const int64_t n = min(((int64_t)max(a.kv_len[b], 0) + (1 << a.page_log2) - 1) >> a.page_log2, a.max_pages), row = b * a.max_pages;
        for (int64_t j = tid; j < n; j += THREADS) a.table_out[row + j] = a.table[row + j];
    }
}
// free_out: {head, free pages so far}.  One tile for a few thousand pages, as the code of four is slow to come (2.6 us, 4.8).
template <int TILES>
__global__ __launch_bounds__(1024) void kv_give_back_kernel(const Books a) {
    const int head = a.free_in[0], count = a.free_in[1], left = a.free_out[1];
    if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) return;   // a refused step: nothing has changed
    const int given = give_back<1024, TILES>(a.shared_out, a.shared_out, a.n_pages, a.ring, head, count);
    if (given > a.n_pages - count) {
        __syncthreads();
        take_back<1024>(a);
    } else if (threadIdx.x == 0) {
        a.free_out[1] = left + given;
    }
}
// the same as the end of a step by one workgroup; go: the step is not refused
template <int THREADS>
__device__ __forceinline__ void give_back_here(const Books &a, const int32_t *counts, bool go, int head, int count, int left) {
    __syncthreads();
    if (!go) {
        for (int i = threadIdx.x; i < a.n_pages; i += THREADS) a.shared_out[i] = counts[i];
        return;
    }
    const int given = give_back<THREADS, 1>(counts, a.shared_out, a.n_pages, a.ring, head, count);
    if (given > a.n_pages - count) {
        __syncthreads();
        take_back<THREADS>(a);
    } else if (threadIdx.x == 0) {
        a.free_out[1] = left + given;
    }
}

template <bool ONE>
__global__ __launch_bounds__(Sizes<ONE>::THREADS) void kv_fork_kernel(const ForkArgs a) {
    constexpr int THREADS = Sizes<ONE>::THREADS;
    __shared__ int n_child[Sizes<ONE>::B], first_child[Sizes<ONE>::B], copy_at[Sizes<ONE>::B];   // copy_at: which of the taken pages, -1: none
    __shared__ uint8_t end[Sizes<ONE>::B];      // the page that a request's length ends in: 0 full, 1 partly filled, 2 and held by another one too
    __shared__ int counts[Sizes<ONE>::PAGES], len_held[ONE ? Sizes<ONE>::B : 1], parent_held[ONE ? Sizes<ONE>::B : 1];
    __shared__ int waves[THREADS / 64];
    const int tid = threadIdx.x, page1 = (1 << a.page_log2) - 1;
    const int64_t capacity = a.max_pages << a.page_log2;
    const int head = a.free_in[0], count = a.free_in[1];
    const bool lead = blockIdx.x == 0;
    auto len_of = [&](int b) { return ONE ? len_held[b] : a.kv_len[b]; };
    auto parent_of = [&](int b) { return ONE ? parent_held[b] : a.parent[b]; };
    auto pages_of = [&](int L) { return (int)(((int64_t)L + page1) >> a.page_log2); };
    for (int b = tid; b < a.B; b += THREADS) {
        n_child[b] = 0, first_child[b] = a.B;
        if constexpr (ONE) len_held[b] = a.kv_len[b], parent_held[b] = a.parent[b];
    }
    if constexpr (ONE)
        for (int i = tid; i < a.n_pages; i += THREADS) counts[i] = max(a.shared[i], 0);
    __syncthreads();
    bool bad = head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages;
    for (int b = tid; b < a.B; b += THREADS) {
        const int p = parent_of(b), L = len_of(b);
        const bool wrong = L < 0 || L > capacity;
        bad |= p < -1 || p >= a.B || wrong;
        if (p >= 0 && p < a.B) {
            atomicAdd(&n_child[p], 1);
            atomicMin(&first_child[p], b);
        }
        int e = 0;
        if (!wrong && (L & page1)) {
            const int id = a.table[(int64_t)b * a.max_pages + pages_of(L) - 1];
            e = (unsigned)id < (unsigned)a.n_pages && (ONE ? counts : a.shared)[id] > 0 ? 2 : 1;
        }
        end[b] = (uint8_t)e;
    }
    bad = __syncthreads_or(bad);
    int need = 0;
    if (!bad)
        for (int b0 = 0; b0 < a.B; b0 += THREADS) {
            const int b = b0 + tid, p = b < a.B ? parent_of(b) : -1;
            const int copied = p >= 0 && end[p] && (b != first_child[p] || end[p] == 2);
            int total;
            const int before = block_scan<THREADS>(copied, waves, total);
            if (b < a.B) copy_at[b] = copied ? need + before : -1;
            need += total;
        }
    __syncthreads();
    const bool go = !bad && need <= count;
    const int head_out = go ? ring_at(head, need, a.n_pages) : head, left = go ? count - need : count;
    if (lead && tid == 0) {
        *a.status = bad ? -1 : go ? 0 : need - count;
        a.free_out[0] = head_out;
        a.free_out[1] = left;                                  // the pages given back come on top
    }
    if (lead)
        for (int b = tid; b < a.B; b += THREADS) {
            const int p = go ? parent_of(b) : b, L = p >= 0 ? len_of(p) : 0;
            const bool copied = go && copy_at[b] >= 0;
            a.kv_len_out[b] = L;
            a.copy_src[b] = copied ? a.table[(int64_t)p * a.max_pages + pages_of(L) - 1] : -1;
            a.copy_dst[b] = copied ? a.ring[ring_at(head, copy_at[b], a.n_pages)] : -1;
        }
    over_table<ONE>(a.B, a.max_pages, [&](int b, int j) {
        // its pages after the call
        const int p = go ? parent_of(b) : b;
        if (p >= 0) {
            const int L = max(len_of(p), 0), n = (int)min((int64_t)pages_of(L), a.max_pages);
            if (j < n) {
                const int at = go && j == n - 1 ? copy_at[b] : -1;
                a.table_out[(int64_t)b * a.max_pages + j] = at >= 0 ? a.ring[ring_at(head, at, a.n_pages)] : a.table[(int64_t)p * a.max_pages + j];
            }
        }
        if (!go) return;
        // the holders of its pages before the call: every copy is one, itself no longer
        const int L = len_of(b), n = pages_of(L), more = n_child[b] - 1;
        if (j < n) {
            const int change = j < L >> a.page_log2 ? more : more < 0 || end[b] == 2 ? -1 : 0;
            const int id = change ? a.table[(int64_t)b * a.max_pages + j] : -1;
            if ((unsigned)id < (unsigned)a.n_pages) atomicAdd((ONE ? counts : a.shared_out) + id, change);
        }
    });
    if constexpr (ONE) give_back_here<THREADS>(a, counts, go, head, count, left);
}

// ---------------------------------------------------------------- requests that lose tokens
struct CompactArgs : Books {
    const int32_t *stay, *cu, *keep;
    int64_t N;
    int32_t *checked;                 // AGQ_KV_CHECKS words behind the new pages in `moves`
};

// do the listed tokens ascend inside their requests?  (cu in LDS)
__device__ __forceinline__ bool listed_wrongly(const CompactArgs &a, const int *cu, int64_t i) {
    const int b = agq_find_row(cu, a.B, (int)i);
    if (i < cu[b] || i >= cu[b + 1]) return false;         // of no request
    const int x = a.keep[i];
    return x >= a.kv_len[b] || x < a.stay[b] || (i > max(cu[b], 0) && x <= a.keep[i - 1]);     // a cu may be anything
}

// the holders' counts, and the check
__global__ __launch_bounds__(512) void kv_compact_check_kernel(const CompactArgs a) {
    __shared__ int cu[kMaxB + 1];
    const int tid = threadIdx.x;
    for (int i = blockIdx.x * 512 + tid; i < a.n_pages; i += gridDim.x * 512) a.shared_out[i] = max(a.shared[i], 0);
    for (int b = tid; b <= a.B; b += 512) cu[b] = a.cu[b];
    __syncthreads();
    bool bad = false;
    if (a.B > 0)
        for (int64_t i = (int64_t)blockIdx.x * 512 + tid; i < a.N; i += (int64_t)gridDim.x * 512) bad |= listed_wrongly(a, cu, i);
    bad = __syncthreads_or(bad);
    if (tid == 0) a.checked[blockIdx.x] = bad;
}

template <bool ONE>
__global__ __launch_bounds__(Sizes<ONE>::THREADS) void kv_compact_kernel(const CompactArgs a, int checked) {
    constexpr int THREADS = Sizes<ONE>::THREADS;
    __shared__ int need_at[Sizes<ONE>::B + 1], same_of[Sizes<ONE>::B], after_of[Sizes<ONE>::B];  // taken pages before, pages that stay, length after
    __shared__ int counts[Sizes<ONE>::PAGES];
    __shared__ int waves[THREADS / 64];
    const int tid = threadIdx.x, page1 = (1 << a.page_log2) - 1;
    const int64_t capacity = a.max_pages << a.page_log2;
    const int head = a.free_in[0], count = a.free_in[1];
    const bool lead = blockIdx.x == 0;
    bool bad = head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages;
    if constexpr (ONE) {
        for (int i = tid; i < a.n_pages; i += THREADS) counts[i] = max(a.shared[i], 0);
        for (int b = tid; b <= a.B; b += THREADS) need_at[b] = a.cu[b];          // for the check
        __syncthreads();
        if (a.B > 0)
            for (int64_t i = tid; i < a.N; i += THREADS) bad |= listed_wrongly(a, need_at, i);
    } else if (tid < checked) {
        bad |= a.checked[tid] != 0;
    }
    for (int b = tid; b < a.B; b += THREADS) {
        const int L = a.kv_len[b], c0 = a.cu[b], c1 = a.cu[b + 1];
        bad |= L < 0 || L > capacity || a.stay[b] < 0 || c0 < 0 || c1 < c0 || c1 > a.N;
    }
    bad = __syncthreads_or(bad);
    auto pages_of = [&](int L) { return (int)(((int64_t)L + page1) >> a.page_log2); };
    int need = 0;
    if (!bad)
        for (int b0 = 0; b0 < a.B; b0 += THREADS) {
            const int b = b0 + tid;
            int mine = 0;
            if (b < a.B) {
                const int L = a.kv_len[b], s = min(a.stay[b], L), n = a.cu[b + 1] - a.cu[b], after = s + n, total = pages_of(after);
                int same = n > 0 ? s >> a.page_log2 : total;
                if (n == 0 && after < L && (after & page1)) {            // cut inside a page, which it will write into
                    const int id = a.table[(int64_t)b * a.max_pages + total - 1];
                    if ((unsigned)id < (unsigned)a.n_pages && a.shared[id] > 0) same = total - 1;
                }
                mine = total - same;
                same_of[b] = same, after_of[b] = after;
            }
            int total;
            const int before = block_scan<THREADS>(mine, waves, total);
            if (b < a.B) need_at[b] = need + before;
            need += total;
        }
    __syncthreads();
    const bool go = !bad && need <= count;
    const int head_out = go ? ring_at(head, need, a.n_pages) : head, left = go ? count - need : count;
    if (lead && tid == 0) {
        *a.status = bad ? -1 : go ? 0 : need - count;
        a.free_out[0] = head_out;
        a.free_out[1] = left;                                  // the pages given back come on top
        a.moves[0] = go ? need : 0;
    }
    if (lead)
        for (int b = tid; b < a.B; b += THREADS) a.kv_len_out[b] = go ? after_of[b] : a.kv_len[b];
    over_table<ONE>(a.B, a.max_pages, [&](int b, int j) {
        const int held = (int)min((int64_t)pages_of(max(a.kv_len[b], 0)), a.max_pages);
        const int same = go ? same_of[b] : held, after = go ? after_of[b] : 0, total = go ? pages_of(after) : held;
        const int old = j < held ? a.table[(int64_t)b * a.max_pages + j] : -1;
        if (j < total) {
            int id = old;
            if (j >= same) {
                const int u = need_at[b] + j - same;
                id = a.ring[ring_at(head, u, a.n_pages)];
                reinterpret_cast<int4 *>(a.moves)[1 + u] = make_int4(b, j, id, min(after - (j << a.page_log2), 1 << a.page_log2));
            }
            a.table_out[(int64_t)b * a.max_pages + j] = id;
        }
        if (j >= same && (unsigned)old < (unsigned)a.n_pages) atomicAdd((ONE ? counts : a.shared_out) + old, -1);
    });
    if constexpr (ONE) give_back_here<THREADS>(a, counts, go, head, count, left);
}

// ---------------------------------------------------------------- the caches of all layers
struct Layers {                       // a launch's arguments
    int8_t *k[AGQ_KV_LAYERS], *v[AGQ_KV_LAYERS], *ke[AGQ_KV_LAYERS], *ve[AGQ_KV_LAYERS];
};

// A workgroup copies 4 KB of each page (its keys, then its values) of `some` entries of the list, in one layer, eight of them at a
// time.  Eight entries, as a wavefront waits for its stores before it has what it loads behind them (224 pages of 8 layers, 117 MB
// written, 58 us with 64 entries to a workgroup, 45 with sixteen, 34 with eight, 3.5 TB/s); more where there would be more than
// eight thousand workgroups, most of which may find nothing to do.
__global__ __launch_bounds__(256) void kv_copy_pages_kernel(const Layers c, const int32_t *src, const int32_t *dst, int n, int some, int n_pages,
                                                            int Hkv, int page_bytes) {
    constexpr int AT_ONCE = 8;
    const int tid = threadIdx.x, lane = tid & 63, layer = blockIdx.y, i = blockIdx.z * some + lane;
    const bool there = lane < some && i < n;
    const int from = there ? src[i] : -1, to = there ? dst[i] : -1;
    unsigned long long todo = __ballot((unsigned)from < (unsigned)n_pages && (unsigned)to < (unsigned)n_pages);
    const int64_t at = ((int64_t)blockIdx.x * 256 + tid) * 16;
    const bool values = at >= page_bytes, mine = at < 2 * (int64_t)page_bytes;
    int8_t *codes = (values ? c.v[layer] : c.k[layer]) + (values ? at - page_bytes : at);
    if (blockIdx.x == 0)
        for (unsigned long long left = todo; left; left &= left - 1) {
            const int e = __ffsll((long long)left) - 1;
            const int64_t s = __builtin_amdgcn_readlane(from, e), d = __builtin_amdgcn_readlane(to, e);
            for (int h = tid; h < Hkv; h += 256) {
                c.ke[layer][d * Hkv + h] = c.ke[layer][s * Hkv + h];
                c.ve[layer][d * Hkv + h] = c.ve[layer][s * Hkv + h];
            }
        }
    if (!mine) return;
    auto next = [&](const int8_t *&from_at, int8_t *&to_at) {
        const int e = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        from_at = codes + (int64_t)__builtin_amdgcn_readlane(from, e) * page_bytes;
        to_at = codes + (int64_t)__builtin_amdgcn_readlane(to, e) * page_bytes;
    };
    for (int left = __popcll(todo); left >= AT_ONCE; left -= AT_ONCE) {
        const int8_t *s[AT_ONCE];
        int8_t *d[AT_ONCE];
        agq_v4i x[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) next(s[j], d[j]);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) x[j] = *reinterpret_cast<const agq_v4i *>(s[j]);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) *reinterpret_cast<agq_v4i *>(d[j]) = x[j];
    }
    while (todo) {
        const int8_t *s;
        int8_t *d;
        next(s, d);
        *reinterpret_cast<uint4 *>(d) = *reinterpret_cast<const uint4 *>(s);
    }
}

// Past the caches: what is moved in all layers is more than they hold when the first layer's attention reads it (8 requests of up to
// 16384 tokens 50 -> 44 us; with two layers only and their attention right behind 69.6 -> 70.3).
__device__ __forceinline__ void store_past(int8_t *p, const uint4 &x) { __builtin_nontemporal_store(__builtin_bit_cast(agq_v4i, x), reinterpret_cast<agq_v4i *>(p)); }

struct MoveArgs {
    const int32_t *moves, *table, *stay, *cu, *keep;
    int64_t max_pages, N;
    int B, layers, Hkv, D, D_log2, page, page_log2, n_pages, most;      // most: new pages that `moves` has room for
};

// An item is a new page of one layer, for one head; a workgroup takes neighbouring items, most of them of one page, whose tokens'
// old places it looks up once.  Tokens of one old page are neighbours in the new one: a run.  Keys are rows, copied 16 bytes at
// a time.  Values lie transposed: lanes are rows d, and a wavefront takes sixteen old tokens of 64 rows, of which it puts those
// that are kept into the new tile in LDS, byte by byte, as which ones they are is the same for all lanes; rows there are an odd
// number of words apart, so that the lanes' bytes are in different banks.
// Bound by memory, in whole old pages: of a page every line is read also where half of its tokens go (8 requests of up to
// 16384 tokens, two layers of 8 heads: 99 MB of kept tokens' codes, 128 MB moved, 34 us, 3.8 TB/s).  Level or slower: the next item's loads
// issued before the tile is written (42 us), kept columns picked by matrix instructions (54), a tile as large as the page needs.
__global__ __launch_bounds__(256) void kv_move_kernel(const Layers c, const MoveArgs a) {
    __shared__ uint32_t run_mask[128][4];                   // which of its tokens a run's old page gives
    __shared__ int run_page[128], run_first[128], run_exp[2][128], run_of[128], slot_of[128];
    __shared__ int n_runs, gaps, top_exp[2];             // gaps: tokens whose old page is not in the cache
    __shared__ uint32_t tile[128 * 33];                     // [D][page + 4] bytes
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t items = (int64_t)min(max(a.moves[0], 0), a.most) * a.layers * a.Hkv, per = (items + gridDim.x - 1) / gridDim.x;
    const int64_t stride = (int64_t)a.Hkv * a.page << a.D_log2;
    const int row = a.page + 4;
    int have = -1, n = 0, to_page = -1;
    for (int64_t item = blockIdx.x * per; item < min((blockIdx.x + 1) * per, items); ++item) {
        const int head = (int)(item % a.Hkv), layer = (int)(item / a.Hkv % a.layers), u = (int)(item / a.Hkv / a.layers);
        if (u != have) {
            have = u;
            const int4 m = reinterpret_cast<const int4 *>(a.moves)[1 + u];      // request, entry, page, tokens
            const int b = min(max(m.x, 0), a.B - 1), j = m.y;
            n = min(max(m.w, 0), a.page), to_page = m.z;
            __syncthreads();                                // the items before are done with the runs
            if (tid < 128) run_mask[tid][0] = run_mask[tid][1] = run_mask[tid][2] = run_mask[tid][3] = 0;
            __syncthreads();
            if (wave == 0) {
                int runs = 0, last = -1, lost = 0;
                for (int t0 = 0; t0 < n; t0 += 64) {
                    const int t = t0 + lane;
                    int id = -1, slot = 0;
                    if (t < n) {
                        const int64_t i = ((int64_t)j << a.page_log2) + t;
                        const int s = a.stay[b];
                        int64_t old = i;
                        if (i >= s) {
                            const int64_t at = a.cu[b] + i - s;
                            old = at >= 0 && at < a.N ? a.keep[at] : -1;
                        }
                        const int64_t entry = old >> a.page_log2;
                        if (old >= 0 && entry < a.max_pages) id = a.table[b * a.max_pages + entry], slot = (int)(old & (a.page - 1));
                        if ((unsigned)id >= (unsigned)a.n_pages) id = -1;
                    }
                    const int before = __shfl_up(id, 1);
                    const bool begins = t < n && (lane == 0 ? t0 == 0 || id != last : id != before);
                    const unsigned long long at = __ballot(begins), upto = at & (~0ull >> (63 - lane));
                    const int r = runs + __popcll(upto) - 1;
                    if (begins) run_page[r] = id, run_first[r] = t;
                    if (t < n) {
                        run_of[t] = r, slot_of[t] = slot;
                        atomicOr(&run_mask[r][slot >> 5], 1u << (slot & 31));
                    }
                    runs += __popcll(at);
                    last = __builtin_amdgcn_readlane(id, 63);
                    lost |= __any(t < n && id < 0);
                }
                if (lane == 0) n_runs = runs, gaps = lost;
            }
            __syncthreads();
        }
        if ((unsigned)to_page >= (unsigned)a.n_pages) continue;
        const int64_t mine = (int64_t)head * a.page << a.D_log2;
        if (tid < 2) top_exp[tid] = -128;
        __syncthreads();                                    // and the item before is done with the exponents and the tile
        const int runs = n_runs;
        for (int i = tid; i < 2 * runs; i += 256) {
            const int v = i >= runs, r = i - v * runs, id = run_page[r];
            const int e = id < 0 ? -128 : (v ? c.ve[layer] : c.ke[layer])[(int64_t)id * a.Hkv + head];
            run_exp[v][r] = e;
            atomicMax(&top_exp[v], e);
        }
        if (n < a.page || gaps)                             // behind the tokens, and where no old page is
            for (int w = tid; w < (a.D * row) >> 2; w += 256) tile[w] = 0;
        __syncthreads();
        const int e_k = top_exp[0], e_v = top_exp[1];
        if (tid < 2) (tid ? c.ve[layer] : c.ke[layer])[(int64_t)to_page * a.Hkv + head] = (int8_t)(tid ? e_v : e_k);
        // values, into the tile
        const int8_t *from_v = c.v[layer] + mine;
        const int halves = a.D >> 6, chunks = a.page >> 4, units = runs * chunks * halves;
        for (int w = wave; w < units; w += 4) {
            const int half = w & (halves - 1), k0 = (w / halves) & (chunks - 1), r = w / halves / chunks, id = run_page[r];
            if (id < 0) continue;
            uint32_t bits = (run_mask[r][k0 >> 1] >> ((k0 & 1) * 16)) & 0xFFFFu;
            bits = __builtin_amdgcn_readfirstlane(bits);
            if (bits == 0) continue;
            int t = run_first[r];
            for (int q = 0; q < k0; ++q) t += __popc((run_mask[r][q >> 1] >> ((q & 1) * 16)) & 0xFFFFu);
            t = __builtin_amdgcn_readfirstlane(t);
            const int d = half * 64 + lane;
            const uint4 x = *reinterpret_cast<const uint4 *>(from_v + id * stride + (d << a.page_log2) + k0 * 16);
            const float down = __builtin_amdgcn_ldexpf(1.0f, run_exp[1][r] - e_v);
            const uint32_t words[4] = {x.x, x.y, x.z, x.w};
            uint8_t *out = reinterpret_cast<uint8_t *>(tile) + d * row;
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (bits >> k & 1) out[t++] = (uint8_t)agq_coarser((int8_t)(words[k >> 2] >> ((k & 3) * 8)), down);
        }
        // keys
        const int8_t *from_k = c.k[layer] + mine;
        int8_t *to_k = c.k[layer] + to_page * stride + mine, *to_v = c.v[layer] + to_page * stride + mine;
        const int per_log2 = a.D_log2 - 4;
        for (int w = tid; w < a.page << per_log2; w += 256) {
            const int t = w >> per_log2, d = (w & ((1 << per_log2) - 1)) * 16, r = t < n ? run_of[t] : 0, id = t < n ? run_page[r] : -1;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (id >= 0) {
                x = *reinterpret_cast<const uint4 *>(from_k + id * stride + (slot_of[t] << a.D_log2) + d);
                const float down = __builtin_amdgcn_ldexpf(1.0f, run_exp[0][r] - e_k);
                if (down != 1.0f) x = make_uint4(agq_coarser4(x.x, down), agq_coarser4(x.y, down), agq_coarser4(x.z, down), agq_coarser4(x.w, down));
            }
            store_past(to_k + (t << a.D_log2) + d, x);
        }
        __syncthreads();
        const int chunk_log2 = a.page_log2 - 4;
        for (int w = tid; w < a.D << chunk_log2; w += 256) {
            const int d = w >> chunk_log2, k = w & (chunks - 1);
            const uint32_t *p = tile + ((d * row) >> 2) + k * 4;
            store_past(to_v + w * 16, make_uint4(p[0], p[1], p[2], p[3]));
        }
    }
}

int log2_of(int64_t v) { return __builtin_ctzll((unsigned long long)v); }
unsigned at_most(int64_t n, int64_t most) { return (unsigned)(n < 1 ? 1 : n > most ? most : n); }

}  // namespace

static Books books_of(const AgqKvPages &p, int32_t *copy_src, int32_t *copy_dst, int32_t *moves) {
    return {p.kv_len, p.table, p.shared, p.free_in, p.ring, p.kv_len_out, p.table_out, p.shared_out, p.free_out, p.status, copy_src, copy_dst, moves,
            p.max_pages, (int)p.B, log2_of(p.page), (int)p.n_pages};
}
static int launch_give_back(const Books &a, hipStream_t st) {
    auto kernel = a.n_pages <= 16384 ? kv_give_back_kernel<1> : kv_give_back_kernel<4>;
    kernel<<<1, 1024, 0, st>>>(a);
    return (int)hipGetLastError();
}

int agq_launch_kv_fork(const AgqKvPages &p, const int32_t *parent, int32_t *copy_src, int32_t *copy_dst, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    const ForkArgs a = {books_of(p, copy_src, copy_dst, nullptr), parent};
    if (agq_kv_one(p.B, p.max_pages, p.n_pages, 0)) {
        kv_fork_kernel<true><<<1, 1024, 0, st>>>(a);
        return (int)hipGetLastError();
    }
    shared_copy_kernel<<<at_most((p.n_pages + 255) / 256, 256), 256, 0, st>>>(p.shared, p.shared_out, (int)p.n_pages);
    if (int err = (int)hipGetLastError()) return err;
    kv_fork_kernel<false><<<at_most(p.B * ((p.max_pages + 511) / 512), 256), 512, 0, st>>>(a);
    if (int err = (int)hipGetLastError()) return err;
    return launch_give_back(a, st);
}

int agq_launch_kv_compact(const AgqKvPages &p, const int32_t *stay, const int32_t *cu, const int32_t *keep, int64_t N, int32_t *moves, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    const CompactArgs a = {books_of(p, nullptr, nullptr, moves), stay, cu, keep, N, moves + 4 + 4 * agq_kv_new_pages(N, p.B, p.page)};
    if (agq_kv_one(p.B, p.max_pages, p.n_pages, N)) {
        kv_compact_kernel<true><<<1, 1024, 0, st>>>(a, 0);
        return (int)hipGetLastError();
    }
    const int64_t work = N > p.n_pages ? N : p.n_pages;
    const unsigned groups = at_most((work + 511) / 512, AGQ_KV_CHECKS);
    kv_compact_check_kernel<<<groups, 512, 0, st>>>(a);
    if (int err = (int)hipGetLastError()) return err;
    kv_compact_kernel<false><<<at_most(p.B * ((p.max_pages + 511) / 512), 256), 512, 0, st>>>(a, (int)groups);
    if (int err = (int)hipGetLastError()) return err;
    return launch_give_back(a, st);
}

static Layers layers_of(const AgqKvLayer *c, int n) {
    Layers l = {};
    for (int i = 0; i < n; ++i) l.k[i] = c[i].k, l.v[i] = c[i].v, l.ke[i] = c[i].k_exp, l.ve[i] = c[i].v_exp;
    return l;
}

int agq_launch_kv_copy_pages(const AgqKvShape &s, const AgqKvLayer *layers, int n_layers, const int32_t *src, const int32_t *dst, int64_t n,
                             void *stream) {
    const int64_t bytes = s.Hkv * s.page * s.D;
    const int64_t slices = (2 * bytes + 4095) / 4096;
    int some = 8;
    while (some < 64 && (n + some - 1) / some * slices * n_layers > 8192) some *= 2;
    const dim3 grid((unsigned)slices, (unsigned)n_layers, (unsigned)((n + some - 1) / some));
    kv_copy_pages_kernel<<<grid, 256, 0, (hipStream_t)stream>>>(layers_of(layers, n_layers), src, dst, (int)n, some, (int)s.n_pages, (int)s.Hkv,
                                                                (int)bytes);
    return (int)hipGetLastError();
}

int agq_launch_kv_move(const AgqKvShape &s, const AgqKvLayer *layers, int n_layers, const int32_t *moves, const int32_t *table, int64_t max_pages,
                       const int32_t *stay, const int32_t *cu, const int32_t *keep, int64_t N, int64_t B, void *stream) {
    const int64_t most = agq_kv_new_pages(N, B, s.page);
    const MoveArgs a = {moves, table, stay, cu, keep, max_pages, N, (int)B, n_layers, (int)s.Hkv, (int)s.D, log2_of(s.D), (int)s.page, log2_of(s.page),
                        (int)s.n_pages, (int)most};
    kv_move_kernel<<<at_most(most * n_layers * s.Hkv, 2048), 256, 0, (hipStream_t)stream>>>(layers_of(layers, n_layers), a);
    return (int)hipGetLastError();
}
