"""The serving calls on the GPU against plain definitions in float64 and whole numbers: the page map and the cache's codes
bit for bit, the attentions within the bound that their roundings allow (oracle/agq_serve_oracle.py)."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import agq_serve_oracle as so  # noqa: E402
from paper_2312_05693_amd import synth  # noqa: E402
from test_gpu_parity import dev, host  # noqa: E402


@pytest.fixture(scope="module")
def agq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2312_05693_amd import binding
    binding.lib()
    return binding


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def rng_of(*key):
    return np.random.default_rng(list(key))


# ------------------------------------------------------------------ the page map

class Pool:
    """Requests with pages already dealt out at random, and the ring of the free ones."""

    def __init__(self, r, lens, page, max_pages, spare, head=None):
        up = -(-np.asarray(lens) // page)
        self.n_pages = int(up.sum()) + spare
        ids = r.permutation(self.n_pages)
        self.table = r.integers(-5, self.n_pages + 5, (len(lens), max_pages)).astype(np.int32)      # what lies behind is anything
        at = 0
        for b, u in enumerate(up):
            self.table[b, :u] = ids[at:at + u]
            at += u
        self.head = int(r.integers(0, self.n_pages)) if head is None else head
        self.ring = np.full(self.n_pages, -1, dtype=np.int32)
        self.ring[(self.head + np.arange(spare)) % self.n_pages] = ids[at:]
        self.state = [self.head, spare]


def check_map(agq, lens, new, page, table, ring, state, T):
    want = so.kv_map(lens, new, table, page, ring, state, T)
    d_table, d_ring = i32(table), i32(ring)
    step = agq.kv_map(i32(lens), i32(new), d_table, page, d_ring, i32(state), T)
    got = (step.kv_len, step.cu_new, step.pos, step.slot, d_table, d_ring, step.free_state, step.status)
    torch.cuda.synchronize()
    for name, g, w in zip(("kv_len", "cu_new", "pos", "slot", "table", "ring", "free_state", "status"), got, want):
        assert np.array_equal(host(g).reshape(-1), np.asarray(w, dtype=np.int32).reshape(-1)), name
    return want


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("B,longest,pad", [(1, 1, 0), (3, 40, 5), (64, 300, 0), (513, 200, 77), (1500, 30, 1)])
def test_map(agq, page, B, longest, pad):
    r = rng_of(page, B)
    lens = r.integers(0, longest + 1, B)
    new = r.choice([-1, 0, 1, 1, 1, page, longest], B)
    most = -(-int((lens + np.maximum(new, 0)).max()) // page) + 1
    pool = Pool(r, lens, page, most, int(np.maximum(new, 0).sum()) // page + B + 3)
    want = check_map(agq, lens, new, page, pool.table, pool.ring, pool.state, int(np.maximum(new, 0).sum()) + pad)
    assert want[-1] == 0


def test_map_long_prompts(agq):
    """tokens, table entries and returned pages shared by many workgroups; the ring wraps around"""
    r = rng_of(1)
    lens, new = np.array([0, 9000, 5, 0, 7000, 0]), np.array([20000, -1, 11000, 0, -1, 1])
    pool = Pool(r, lens, 16, 1300, 2000, head=1900)
    assert check_map(agq, lens, new, 16, pool.table, pool.ring, pool.state, 31001)[-1] == 0


@pytest.mark.parametrize("what", ["short", "long", "negative", "minus2", "tokens", "head", "count", "returns"])
def test_map_leaves_a_step_out(agq, what):
    r = rng_of(2)
    lens, new, T, spare = np.array([30, 0, 64, 7]), np.array([1, 70, -1, 3]), 74, 6
    pool = Pool(r, lens, 16, 5, spare)
    if what == "short":
        pool.state[1] = 3
    elif what == "long":
        new[1] = 81
    elif what == "negative":
        lens[0] = -1
    elif what == "minus2":
        new[2] = -2
    elif what == "tokens":
        T = 73
    elif what == "head":
        pool.state[0] = pool.n_pages
    elif what == "count":
        pool.state[1] = -1
    else:
        pool.state[1] = pool.n_pages - 1
    status = check_map(agq, lens, new, 16, pool.table, pool.ring, pool.state, T)[-1]
    assert status == (2 if what == "short" else -1)


def test_map_sums_beyond_32_bits_are_refused(agq):
    """4000 requests that ask for 2^30 tokens each"""
    B = 4000
    check_map(agq, [0] * B, [1 << 30] * B, 128, np.zeros((B, 1), np.int32), np.arange(9, dtype=np.int32), [0, 9], 50)
    d_table = torch.zeros(1, (1 << 31) // 128 - 1, dtype=torch.int32, device="cuda")
    step = agq.kv_map(i32([0]), i32([(1 << 31) - 129]), d_table, 128, i32(np.arange(9)), i32([0, 9]), 4)
    assert host(step.status)[0] == -1 and (host(step.slot) == -1).all()


def test_map_nothing_new(agq):
    pool = Pool(rng_of(3), [17, 1], 16, 2, 1)
    assert check_map(agq, [17, 1], [-1, 0], 16, pool.table, pool.ring, pool.state, 0)[-1] == 0
    check_map(agq, [], [], 16, np.zeros((0, 3), np.int32), pool.ring, pool.state, 4)


def test_map_page_number_outside_the_cache(agq):
    pool = Pool(rng_of(4), [17, 5], 16, 3, 4)
    pool.table[0, 1], pool.table[1, 0] = pool.n_pages, -3
    want = check_map(agq, [17, 5], [2, 1], 16, pool.table, pool.ring, pool.state, 3)
    assert want[3] == [-1, -1, -1]
    with pytest.raises(agq.AgqError):
        agq.kv_map(i32([0]), i32([1]), i32([[0]]), 17, i32([0]), i32([0, 1]), 1)
    step = agq.kv_map(i32([0]), i32([1]), i32([[0]]), 16, i32([0]), i32([0, 1]), 1)
    with pytest.raises(agq.AgqError):       # the lengths would be overwritten while they are read
        agq.kv_map(step.kv_len, i32([1]), i32([[0]]), 16, i32([0]), i32([0, 1]), 1, out=step)


def test_map_many_steps(agq):
    """a server's life: requests come, grow and go, the lengths and the ring's state swapped from step to step"""
    r, B, page, n_pages = rng_of(5), 20, 16, 90
    lens, table, ring, state = [0] * B, np.full((B, 12), -1, np.int32), r.permutation(n_pages).astype(np.int32), [0, n_pages]
    d_table, d_ring = i32(table), i32(ring)
    cur = (i32(lens), i32(state))
    for n in range(40):
        new = [int(r.integers(1, 60)) if L == 0 and r.random() < 0.3 else 0 if L == 0 else -1 if L > 150 or r.random() < 0.05 else 1 for L in lens]
        T = sum(x for x in new if x > 0)
        lens, cu, pos, slot, table, ring, state, status = so.kv_map(lens, new, table, page, ring, state, T)
        step = agq.kv_map(cur[0], i32(new), d_table, page, d_ring, cur[1], T)
        cur = (step.kv_len, step.free_state)
        for g, w in ((step.kv_len, lens), (step.pos, pos), (step.slot, slot), (d_table, table), (d_ring, ring), (step.free_state, state),
                     (step.status, [status])):
            assert np.array_equal(host(g).reshape(-1), np.asarray(w, np.int32).reshape(-1)), n


# ------------------------------------------------------------------ writing into the cache

def random_cache(r, n_pages, Hkv, page, D, lo=-7, hi=-4):
    k = r.integers(-127, 128, (n_pages, Hkv, page, D)).astype(np.int8)
    v = r.integers(-127, 128, (n_pages, Hkv, D, page)).astype(np.int8)
    return k, v, r.integers(lo, hi + 1, (n_pages, Hkv)).astype(np.int8), r.integers(lo, hi + 1, (n_pages, Hkv)).astype(np.int8)


def random_slots(r, past, new, page, n_pages, pad):
    """slots and positions of requests with random pages, `pad` tokens without a slot behind them"""
    ids, slot, pos = list(r.permutation(n_pages)), [], []
    for p0, n in zip(past, new):
        pages = [ids.pop() for _ in range(-(-(p0 + n) // page))]
        pos += range(p0, p0 + n)
        slot += [pages[p // page] * page + p % page for p in range(p0, p0 + n)]
    return np.array(slot + [-1] * pad, np.int32), np.array(pos + [0] * pad, np.int32)


def check_append(agq, r, T, Hq, Hkv, D, page, slot, pos, n_pages, x=None, rope=True, cache=None, fused=True):
    H = Hq + 2 * Hkv
    x = (r.standard_normal((T, H, D)) * np.where(r.random((T, H, D)) < 0.01, 20, 1)).astype(np.float16) if x is None else x
    k_c, v_c, k_e, v_e = random_cache(r, n_pages, Hkv, page, D) if cache is None else cache
    cos, sin = synth.rope_tables(max(int(pos.max(initial=0)), 1), D)       # the last position is beyond the table
    d = [dev(a) for a in (k_c, v_c, k_e, v_e)]
    xd = dev(x)
    q, k, v = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q_out, k_out = torch.full((T, Hq, D), 7.0, dtype=torch.float16, device="cuda"), torch.full((T, Hkv, D), 7.0, dtype=torch.float16, device="cuda")
    if rope:
        got_q, got_k = agq.kv_append(k, v, i32(slot), *d, q=q if Hq else None, pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin),
                                     q_out=q_out if Hq else None, k_out=k_out)
        want_k = so.rotate(x[:, Hq:Hq + Hkv], pos, cos, sin)
        on = ((slot >= 0) & (slot < n_pages * page))[:, None, None]
        sev = np.float16(7.0)
        if Hq:
            assert np.array_equal(host(got_q).view(np.uint16), np.where(on, so.rotate(x[:, :Hq], pos, cos, sin), sev).view(np.uint16))
        assert np.array_equal(host(got_k).view(np.uint16), np.where(on, want_k, sev).view(np.uint16))
    else:
        assert agq.kv_append(k, v, i32(slot), *d) == (None, None)
        want_k = x[:, Hq:Hq + Hkv]
    kc, ke = so.kv_append(want_k, slot, k_c, k_e, False)
    vc, ve = so.kv_append(x[:, Hq + Hkv:], slot, v_c, v_e, True)
    torch.cuda.synchronize()
    for name, g, w in zip(("k", "v", "k_exp", "v_exp"), d, (kc, vc, ke, ve)):
        assert np.array_equal(host(g), w), name
    return d


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 3, 3), (128, 8, 2), (128, 0, 1)])
@pytest.mark.parametrize("past,new,pad", [([0], [1], 0), ([5, 0, 127, 16], [1, 1, 1, 1], 2), ([0, 3, 30], [200, 77, 131], 3), ([63, 15], [1, 2], 0)])
def test_append(agq, page, D, Hq, Hkv, past, new, pad):
    r = rng_of(page, D, len(new), sum(new))
    n_pages = sum(-(-(p + n) // page) for p, n in zip(past, new)) + 3
    slot, pos = random_slots(r, past, new, page, n_pages, pad)
    check_append(agq, r, len(slot), Hq, Hkv, D, page, slot, pos, n_pages)


def test_append_many_tokens(agq):
    """workgroups that take several runs each: runs across their chunks, tokens without a slot in between"""
    r = rng_of(6)
    new = list(r.integers(1, 90, 60))
    past = list(r.integers(0, 40, 60))
    slot, pos = random_slots(r, past, new, 16, 700, 9)
    cut = int(np.cumsum(new)[30])
    slot, pos = np.concatenate([slot[:cut], [-1, -1, 1 << 30], slot[cut:]]).astype(np.int32), np.concatenate([pos[:cut], [0, 0, 0], pos[cut:]]).astype(np.int32)
    check_append(agq, r, len(slot), 4, 12, 64, 16, slot, pos, 700)


@pytest.mark.parametrize("rope,fused", [(False, True), (True, False)])
def test_append_forms(agq, rope, fused):
    r = rng_of(7)
    slot, pos = random_slots(r, [3, 0], [20, 9], 16, 8, 1)
    check_append(agq, r, 30, 0 if not rope else 4, 2, 64, 16, slot, pos, 8, rope=rope, fused=fused)


def test_append_token_by_token_and_scales(agq):
    """a page filled one token at a time: scales that grow, shrinking values that do not lower them, zeros, infinities, the
    smallest and largest values; ties of the codes that become coarser"""
    r, page, D = rng_of(8), 16, 64
    cache = random_cache(r, 3, 2, page, D)
    size = [0.0, 2.0 ** -24, 2.0 ** -14, 1e-3, 0.5, 0.4, 126.9, 127.0, 127.1, 1.0, 0.0, 65504.0, np.inf, 3.0, 1.0, 2.0]
    for off, top in enumerate(size):
        x = np.clip(r.standard_normal((1, 4, D)), -1, 1).astype(np.float16)
        x = np.zeros_like(x) if top == 0 else (x * np.float16(min(top, 1000.0))).astype(np.float16)
        x[0, :, 5] = top
        x[0, 1, 6] = -top
        d = check_append(agq, r, 1, 0, 2, D, page, np.array([page + off], np.int32), np.array([off], np.int32), 3, x=x, rope=False, cache=cache)
        cache = tuple(host(t).copy() for t in d)
    assert (cache[3][1] == 10).all()


def test_append_in_place(agq):
    r, T, Hq, Hkv, D = rng_of(9), 21, 4, 2, 128
    slot, pos = random_slots(r, [4], [T], 32, 2, 0)
    x = r.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float16)
    cos, sin = synth.rope_tables(64, D)
    cache = random_cache(r, 2, Hkv, 32, D)
    a, b = [dev(c) for c in cache], [dev(c) for c in cache]
    xd, yd = dev(x), dev(x)
    part = lambda t: (t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:])
    q, k, v = part(xd)
    rest = dict(pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin))
    want_q, want_k = agq.kv_append(k, v, i32(slot), *a, q=q, **rest)
    q, k, v = part(yd)
    agq.kv_append(k, v, i32(slot), *b, q=q, q_out=q, k_out=k, **rest)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and all(torch.equal(s, t) for s, t in zip(a, b))


# ------------------------------------------------------------------ attention over packed prompts

def ramp(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def check_packed(agq, q, k, v, cu_q, cu_k, causal=True, scale=None, parts=None, finite=True):
    """q, k, v numpy fp16; parts: the device tensors to call with (the same values), q's first"""
    dq, dk, dv = parts or (dev(q), dev(k), dev(v))
    o = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    agq.attn_packed(dq, dk, dv, i32(cu_q), i32(cu_k), causal=causal, scale=scale, o=o)
    got, group = host(o).astype(np.float64), q.shape[1] // k.shape[1]
    for b in range(len(cu_q) - 1):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        for h in range(q.shape[1]):
            kk, vv = (t[cu_k[b]:cu_k[b + 1], h // group].astype(np.float64) for t in (k, v))
            want, bound = so.attention(q[cu_q[b]:cu_q[b + 1], h].astype(np.float64), kk, vv, m - n, causal, scale)
            g = got[cu_q[b]:cu_q[b + 1], h]
            ok = np.isfinite(want)
            assert finite is False or ok.all()
            assert np.array_equal(ok, np.isfinite(g)), (b, h)
            off = np.abs(g - np.where(ok, want, 0))[ok] - np.where(ok, bound, 0)[ok]
            assert off.max(initial=-1.0) <= 0, (b, h, off.max())
    rows = np.zeros(q.shape[0], bool)
    for b in range(len(cu_q) - 1):
        rows[cu_q[b]:cu_q[b + 1]] = True
    assert (got[~rows] == 7.0).all()                     # rows of no sequence stay as they were
    return got


def random_qkv(r, Tq, Tk, Hq, Hkv, D, big=1.5):
    return ((r.standard_normal((Tq, Hq, D)) * big).astype(np.float16), r.standard_normal((Tk, Hkv, D)).astype(np.float16),
            r.standard_normal((Tk, Hkv, D)).astype(np.float16))


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 2, 2), (128, 2, 1), (128, 5, 1), (64, 8, 2)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[1], [2, 0, 1, 31, 32, 33], [63, 64, 65], [127, 128, 129], [300, 1, 257]])
def test_packed(agq, D, Hq, Hkv, causal, lens):
    r = rng_of(D, Hq, causal, sum(lens))
    q, k, v = random_qkv(r, sum(lens), sum(lens), Hq, Hkv, D)
    check_packed(agq, q, k, v, ramp(lens), ramp(lens), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [([5], [300]), ([130, 1, 40], [131, 500, 40]), ([200, 70, 3], [130, 0, 1]), ([0, 129], [77, 64])])
def test_packed_other_key_lengths(agq, causal, n, m):
    """parts of prompts (more keys than queries), and queries before the first key, which see nothing and come out as 0"""
    r = rng_of(11, sum(n), sum(m))
    q, k, v = random_qkv(r, sum(n), sum(m), 4, 2, 128)
    got = check_packed(agq, q, k, v, ramp(n), ramp(m), causal)
    for b in range(len(n)):
        none = max(0, n[b] - m[b]) if causal else (n[b] if m[b] == 0 else 0)
        assert (got[ramp(n)[b]:ramp(n)[b] + none] == 0).all()


def test_packed_many_sequences(agq):
    """more sequences than a wavefront has lanes"""
    lens = list(rng_of(12).integers(0, 40, 150))
    q, k, v = random_qkv(rng_of(13), sum(lens), sum(lens), 2, 1, 64)
    check_packed(agq, q, k, v, ramp(lens), ramp(lens))


def test_packed_long(agq):
    q, k, v = random_qkv(rng_of(14), 70, 5000, 1, 1, 128)
    check_packed(agq, q, k, v, ramp([70]), ramp([5000]))
    q, k, v = random_qkv(rng_of(15), 1100, 1100, 1, 1, 64)
    check_packed(agq, q, k, v, ramp([1100]), ramp([1100]))


@pytest.mark.parametrize("D", [64, 128])
def test_packed_padding_strides_and_values_that_nobody_sees(agq, D):
    """parts of one projection's output; infinities and NaN behind the sequences, between them and after the diagonal"""
    r, lens, Hq, Hkv = rng_of(16), [40, 100, 65], 4, 2
    cu = ramp(lens) + 3                                    # rows 0-2 belong to nobody, nor do the last ones
    T = int(cu[-1]) + 9
    x = r.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float16)
    x[:3] = np.nan
    x[cu[-1]:] = np.inf
    x[cu[1] - 1, Hq:] = np.nan                             # the last key and value of a sequence: only its last query sees them
    x[cu[1] + 70, Hq + Hkv:, 5] = -np.inf                  # a value of the second sequence, seen from row 70 on
    x[cu[1] + 90, Hq + Hkv:, 5] = np.inf                   # and its opposite
    x[cu[2] + 64, Hq:Hq + Hkv] = np.inf
    xd = dev(x)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    check_packed(agq, q, k, v, cu, cu, parts=(xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]), finite=False)


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 2, 1), (64, 4, 4)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [([100], [3000]), ([1, 130, 0, 7], [2500, 4000, 9, 100]), ([1500], [1400])])
def test_packed_shared_keys(agq, D, Hq, Hkv, causal, n, m):
    """few queries, many keys: workgroups share the keys of a tile; sequences longer and shorter than the average, rows
    that see nothing, an infinity and a NaN that nobody sees; a workspace full of NaN"""
    r = rng_of(19, D, sum(n))
    q, k, v = random_qkv(r, sum(n), sum(m), Hq, Hkv, D)
    need = agq.attn_packed_workspace_bytes(sum(n), Hq, sum(m), Hkv, D, len(n))
    assert need > 0
    got = check_packed(agq, q, k, v, ramp(n), ramp(m), causal)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    again = agq.attn_packed(dev(q), dev(k), dev(v), i32(ramp(n)), i32(ramp(m)), causal=causal, workspace=ws)
    assert np.array_equal(host(again).astype(np.float64), got)
    if causal and n[0] > 1 and m[0] > n[0]:
        v[m[0] - 1] = np.nan
        v[m[0] - 2, 0, 3] = np.inf
        check_packed(agq, q, k, v, ramp(n), ramp(m), causal, finite=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [(40, 40), (200, 200), (300, 333), (20, 3000)])
def test_packed_infinities_that_are_seen(agq, D, causal, n, m):
    """an infinity among the values gives infinities of its sign in its column, a NaN or two opposite ones NaN"""
    r = rng_of(20, D, n)
    q, k, v = random_qkv(r, n, m, 2, 1, D)
    v[0, 0, 3], v[7, 0, 5], v[33, 0, 9], v[35, 0, 9], v[m - 1, 0, 11], v[1, 0, 20] = np.inf, -np.inf, np.inf, -np.inf, np.inf, np.nan
    check_packed(agq, q, k, v, ramp([n]), ramp([m]), causal, finite=False)
    o = host(agq.attn_packed(dev(q), dev(k), dev(v), i32(ramp([n])), i32(ramp([m])), causal=causal)).astype(np.float64)
    for i in range(n):
        keys = m - n + i + 1 if causal else m
        assert (o[i, :, 3] == np.inf).all() and (keys <= 7 or (o[i, :, 5] == -np.inf).all())
        assert keys <= 33 or (np.isnan(o[i, :, 9]).all() if keys > 35 else (o[i, :, 9] == np.inf).all())
        assert keys < m or (o[i, :, 11] == np.inf).all()


@pytest.mark.parametrize("D,tokens,Hq,Hkv", [(128, 1100, 40, 40), (64, 1400, 24, 8), (128, 2300, 33, 11)])
def test_packed_one_prompt_of_many_workgroups(agq, D, tokens, Hq, Hkv):
    """more workgroups than CUs, which are taken in another order then: every row of every head against the same head alone"""
    r = rng_of(25, D, tokens)
    q, k, v = (dev(x) for x in random_qkv(r, tokens, tokens, Hq, Hkv, D))
    cu = i32([0, tokens])
    o = torch.full((tokens, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    agq.attn_packed(q, k, v, cu, cu, o=o)
    for h in range(Hq):
        kv = h // (Hq // Hkv)
        alone = agq.attn_packed(q[:, h:h + 1], k[:, kv:kv + 1], v[:, kv:kv + 1], cu, cu,
                                workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
        assert ((o[:, h:h + 1].double() - alone.double()).abs() <= 2.0 ** -9 * alone.double().abs() + 2.0 ** -8).all(), h
    check_packed(agq, *(host(x[:, :1]) for x in (q, k, v)), ramp([tokens]), ramp([tokens]))


def test_packed_scale_and_large_scores(agq):
    """one key that takes all; scores in the thousands; thousands of faint keys under a loud one"""
    r = rng_of(17)
    q, k, v = random_qkv(r, 200, 200, 1, 1, 64, big=30.0)
    check_packed(agq, q, k, v, ramp([200]), ramp([200]), scale=2.0)
    check_packed(agq, q, k, v, ramp([200]), ramp([200]), scale=1e-6)
    q, k, v = np.full((3, 1, 64), 1.0, np.float16), np.full((4000, 1, 64), -0.125, np.float16), np.abs(random_qkv(r, 1, 4000, 1, 1, 64)[2])
    k[5] = 0.125                                           # exp(-16 / 1) beside it: 4000 of 1e-7
    check_packed(agq, q, k, v, ramp([3]), ramp([4000]), scale=1.0)


def test_packed_offsets_outside_the_tensors(agq):
    """offsets are taken into the tensors' bounds: sequences that end behind them are cut"""
    r = rng_of(18)
    q, k, v = random_qkv(r, 50, 60, 2, 2, 64)
    o = torch.full((50, 2, 64), 7.0, dtype=torch.float16, device="cuda")
    agq.attn_packed(dev(q), dev(k), dev(v), i32([0, 20, 1 << 30]), i32([-5, 30, 1 << 30]), causal=False, o=o)
    want = torch.empty_like(o)
    agq.attn_packed(dev(q), dev(k), dev(v), i32([0, 20, 50]), i32([0, 30, 60]), causal=False, o=want)
    assert torch.equal(o, want)


# ------------------------------------------------------------------ attention over the cache

def make_pages(r, lens, page, extra=2):
    up = [-(-int(L) // page) for L in lens]
    n_pages = sum(up) + extra
    ids, at = r.permutation(n_pages), 0
    table = np.full((len(lens), max(max(up), 1)), -1, np.int32)
    for b, u in enumerate(up):
        table[b, :u] = ids[at:at + u]
        at += u
    return table, n_pages


def check_cache(agq, q, cu_q, lens, table, cache, max_q=None, max_kv=None, scale=None, workspace=None):
    n = np.diff(cu_q)
    o = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    agq.attn_kv(dev(q), i32(cu_q), i32(lens), i32(table), *(dev(c) for c in cache), int(n.max()) if max_q is None else max_q,
                int(max(lens)) if max_kv is None else max_kv, scale=scale, o=o, workspace=workspace)
    got, (k_c, v_c, k_e, v_e) = host(o).astype(np.float64), cache
    Hkv, group = k_c.shape[1], q.shape[1] // k_c.shape[1]
    page = k_c.shape[2]
    rows = np.zeros(q.shape[0], bool)
    for b in range(len(lens)):
        L = min(max(int(lens[b]), 0), table.shape[1] * page)
        rows[cu_q[b]:cu_q[b + 1]] = True
        for h in range(Hkv):
            k, there = so.cache_rows(k_c, k_e, table[b], L, h, False)
            v, _ = so.cache_rows(v_c, v_e, table[b], L, h, True)
            for x in range(group):
                hh = h * group + x
                want, bound = so.attention(q[cu_q[b]:cu_q[b + 1], hh].astype(np.float64), k, v, L - int(n[b]), True, scale, there)
                g = got[cu_q[b]:cu_q[b + 1], hh]
                assert np.isfinite(g).all() and (np.abs(g - want) <= bound).all(), (b, hh, (np.abs(g - want) - bound).max())
    assert (got[~rows] == 7.0).all()
    return got


def random_q(r, T, Hq, D):
    return (r.standard_normal((T, Hq, D)) * 1.5).astype(np.float16)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 2, 2), (128, 8, 2), (128, 5, 1), (64, 17, 1), (128, 40, 1)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 15, 16, 17], [63, 64, 65, 130], [700]])
def test_cache(agq, page, D, Hq, Hkv, lens):
    r = rng_of(page, D, Hq, sum(lens))
    table, n_pages = make_pages(r, lens, page)
    q = random_q(r, len(lens) + 2, Hq, D)
    cu = np.arange(len(lens) + 1, dtype=np.int32) + 1       # a row of nobody in front and one behind
    check_cache(agq, q, cu, lens, table, random_cache(r, n_pages, Hkv, page, D))


@pytest.mark.parametrize("n,lens", [([3, 1, 0, 5], [3, 200, 9, 4]), ([8, 8], [64, 400]), ([70], [100]), ([40, 2], [20, 0])])
@pytest.mark.parametrize("max_q", [None, 1])
def test_cache_several_tokens(agq, n, lens, max_q):
    """a draft's tokens, a prompt's part, more new tokens than the cache holds; more of them than max_q says"""
    r = rng_of(21, sum(n))
    table, n_pages = make_pages(r, lens, 16)
    check_cache(agq, random_q(r, sum(n), 6, 64), ramp(n), lens, table, random_cache(r, n_pages, 2, 16, 64), max_q=max_q)


@pytest.mark.parametrize("lens,max_kv", [([20000, 3, 0, 9000], 20000), ([16383, 16384, 16385], 20000), ([30000, 70], 8200), ([9000], 200000),
                                         ([0, 0, 8000, 1, 0, 5000, 257, 256], 8192)])
@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 4, 1, 64), (64, 6, 2, 16)])
def test_cache_pieces_by_the_lengths(agq, lens, max_kv, D, Hq, Hkv, page):
    """few requests with long caches: the device chooses the pieces; empty requests, one long one, longer than max_kv"""
    r, B = rng_of(26, sum(lens), D), len(lens)
    table, n_pages = make_pages(r, lens, page)
    assert agq.attn_kv_workspace_bytes(B, Hq, Hkv, D, B, 1, max_kv) > 0
    check_cache(agq, random_q(r, B, Hq, D), ramp([1] * B), lens, table, random_cache(r, n_pages, Hkv, page, D), max_kv=max_kv)


@pytest.mark.parametrize("lens,max_kv", [([20000, 9, 6, 9000], 60000), ([16383, 16384, 16385], 60000), ([90000, 70], 82000), ([9000], 200000),
                                         ([0, 0, 8000, 1, 0, 5000, 257, 256], 24000), ([1] * 40 + [3000] * 24, 4096)])
@pytest.mark.parametrize("n,D,Hq,Hkv,page", [(1, 128, 4, 1, 64), (1, 64, 6, 2, 16), (6, 128, 4, 1, 32), (9, 64, 6, 2, 128)])
def test_cache_one_piece_per_cu(agq, lens, max_kv, n, D, Hq, Hkv, page):
    """few requests with long caches, one or two tiles of rows: the device chooses the pieces; requests that are empty, that hold fewer
    tokens than are new, or more than max_kv"""
    r, B = rng_of(27, sum(lens), D, n), len(lens)
    table, n_pages = make_pages(r, lens, page)
    need = agq.attn_kv_workspace_bytes(n * B, Hq, Hkv, D, B, n, max_kv)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")                                                     # NaN
    check_cache(agq, random_q(r, n * B, Hq, D), ramp([n] * B), lens, table, random_cache(r, n_pages, Hkv, page, D), max_kv=max_kv, workspace=ws)


def test_cache_shared_keys_no_new_tokens_expected(agq):
    """max_q = 0 with tokens all the same"""
    r, lens = rng_of(24), [3000, 500]
    table, n_pages = make_pages(r, lens, 32)
    assert agq.attn_kv_workspace_bytes(2, 4, 2, 64, 2, 0, 60000) > 0
    check_cache(agq, random_q(r, 2, 4, 64), ramp([1, 1]), lens, table, random_cache(r, n_pages, 2, 32, 64), max_q=0, max_kv=60000)


@pytest.mark.parametrize("lens,max_kv", [([9000], None), ([5000, 3, 0, 1700], None), ([2600, 4100], 1500), ([600], 60000)])
@pytest.mark.parametrize("n", [1, 3])
def test_cache_shared_keys(agq, lens, max_kv, n):
    """the keys of a request shared by several workgroups and joined; longer and shorter than max_kv says"""
    r = rng_of(22, sum(lens), n)
    table, n_pages = make_pages(r, lens, 64)
    B = len(lens)
    T, most = n * B, max(lens) if max_kv is None else max_kv
    assert agq.attn_kv_workspace_bytes(T, 4, 1, 128, B, n, most) > 0
    ws = torch.full((agq.attn_kv_workspace_bytes(T, 4, 1, 128, B, n, most),), 255, dtype=torch.uint8, device="cuda")     # NaN
    check_cache(agq, random_q(r, T, 4, 128), ramp([n] * B), lens, table, random_cache(r, n_pages, 1, 64, 128), max_kv=most, workspace=ws)


def test_cache_scales_far_apart(agq):
    """pages whose scales differ by all that exponents allow, for keys and values; a whole row's weight on the finest page"""
    r, page, D = rng_of(23), 16, 64
    lens = [200, 64]
    table, n_pages = make_pages(r, lens, page)
    k, v, ke, ve = random_cache(r, n_pages, 1, page, D)
    ke[:] = -9
    ve[:] = r.integers(-30, 11, ve.shape)
    v[ve > 8] = np.sign(v[ve > 8]) * 3                       # the largest scales hold no more than fp16's range
    check_cache(agq, random_q(r, 2, 2, D), ramp([1, 1]), lens, table, (k, v, ke, ve))
    ke[:] = r.integers(-30, -3, ke.shape)
    check_cache(agq, random_q(r, 2, 2, D), ramp([1, 1]), lens, table, (k, v, ke, ve), scale=0.5)


def test_cache_pages_outside(agq):
    """page numbers outside the cache: their tokens are left out, wherever they stand"""
    r, page = rng_of(24), 16
    lens = [100, 40, 20]
    table, n_pages = make_pages(r, lens, page)
    table[0, 3], table[0, 0], table[1, 1], table[2, :2] = -1, n_pages, 1 << 30, [-7, n_pages + 9]
    got = check_cache(agq, random_q(r, 3, 4, 128), ramp([1, 1, 1]), lens, table, random_cache(r, n_pages, 2, page, 128))
    assert (got[2] == 0).all()
    # a length beyond the table's row is cut to it, a negative one is none
    check_cache(agq, random_q(r, 3, 4, 128), ramp([1, 1, 1]), [1000, -5, 112], table, random_cache(r, n_pages, 2, page, 128), max_kv=64)


def test_cache_beyond_32_bits(agq):
    """pages whose bytes lie behind 2^31 and 2^32"""
    page, Hkv, D = 128, 8, 128
    n_pages = (1 << 32) // (page * Hkv * D) + 4
    k, v = torch.zeros(n_pages, Hkv, page, D, dtype=torch.int8, device="cuda"), torch.zeros(n_pages, Hkv, D, page, dtype=torch.int8, device="cuda")
    ke, ve = (torch.zeros(n_pages, Hkv, dtype=torch.int8, device="cuda") for _ in range(2))
    r = rng_of(25)
    use = [n_pages - 1, (1 << 31) // (page * Hkv * D), 0]
    small = random_cache(r, 3, Hkv, page, D)
    x = r.standard_normal((3 * page, 3 * Hkv, D)).astype(np.float16)
    slot = np.concatenate([np.arange(page) + u * page for u in use]).astype(np.int32)
    xd = dev(x)
    agq.kv_append(xd[:, Hkv:2 * Hkv], xd[:, 2 * Hkv:], i32(slot), k, v, ke, ve)
    near = (np.arange(3 * page)).astype(np.int32)
    kc, kx = so.kv_append(x[:, Hkv:2 * Hkv], near, small[0], small[2], False)
    vc, vx = so.kv_append(x[:, 2 * Hkv:], near, small[1], small[3], True)
    for big, want in ((k, kc), (v, vc), (ke, kx), (ve, vx)):
        assert np.array_equal(host(big[use]), want)
    o = agq.attn_kv(xd[:1, :Hkv], i32([0, 1]), i32([3 * page - 5]), i32([use]), k, v, ke, ve, 1, 3 * page)
    near = agq.attn_kv(xd[:1, :Hkv], i32([0, 1]), i32([3 * page - 5]), i32([[0, 1, 2]]), dev(kc), dev(vc), dev(kx), dev(vx), 1, 3 * page)
    assert torch.equal(o, near)


# ------------------------------------------------------------------ together, as a server runs them

class Server:
    """One layer's cache and its state on the device; prompts through attn_packed, generation through attn_kv."""

    def __init__(self, agq, B, page, n_pages, Hq, Hkv, D, rows=512):
        self.agq, self.page, self.shape = agq, page, (Hq, Hkv, D)
        dims = dict(dtype=torch.int8, device="cuda")
        self.cache = [torch.zeros(n_pages, Hkv, page, D, **dims), torch.zeros(n_pages, Hkv, D, page, **dims), torch.zeros(n_pages, Hkv, **dims),
                      torch.zeros(n_pages, Hkv, **dims)]
        self.table, self.ring = i32(np.full((B, n_pages), -1)), i32(np.arange(n_pages))
        self.kv_len, self.free = i32([0] * B), i32([0, n_pages])
        self.rope = [dev(t) for t in synth.rope_tables(rows, D)]

    def step(self, qkv, new, max_kv, prompt=False, out=None):
        agq, (Hq, Hkv, D) = self.agq, self.shape
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st = agq.kv_map(self.kv_len, new, self.table, self.page, self.ring, self.free, qkv.shape[0], out=out)
        q, k = agq.kv_append(k, v, st.slot, *self.cache, q=q, pos=st.pos, rope_cos=self.rope[0], rope_sin=self.rope[1])
        a = agq.attn_kv(q, st.cu_new, st.kv_len, self.table, *self.cache, 1, max_kv)
        o = agq.attn_packed(q, k, v, st.cu_new, st.cu_new) if prompt else a
        self.kv_len, self.free = st.kv_len, st.free_state
        return o, a, st


@pytest.mark.parametrize("D,Hq,Hkv,page", [(64, 4, 4, 16), (128, 8, 2, 32)])
def test_prompt_then_generation(agq, D, Hq, Hkv, page):
    """prompts into the cache, then tokens: what the cache gives for a prompt is what the fp16 keys and values give, up to
    the codes' rounding, and every step's output is the float64 attention of the cache's contents"""
    r, B = rng_of(31, D), 3
    s = Server(agq, B, page, 40, Hq, Hkv, D)
    lens = [50, 1, 97]
    x = (r.standard_normal((sum(lens), Hq + 2 * Hkv, D))).astype(np.float16)
    o, a, st = s.step(dev(x), i32(lens), 128, prompt=True)
    assert host(st.status)[0] == 0
    # a code is off by half a step of 2^e, 127 * 2^e below twice the largest value (5): 5 / 127 for a key's or value's entry
    # at most; scores move by |q|_1 / sqrt(D) times that, weights by e^2 of it, the values by their own half step
    q1 = np.abs(so.rotate(x[:, :Hq], host(st.pos), *(host(t) for t in s.rope)).astype(np.float64)).sum(-1).max()
    step = np.abs(x).max().astype(np.float64) * 2 ** 0.5 / 127
    worst = np.exp(2 * step * q1 / D ** 0.5) - 1
    assert np.abs(host(o).astype(np.float64) - host(a)).max() <= worst * 2 * np.abs(x).max() + step
    total = list(lens)
    for n in range(4):
        new = [1, 1, 1] if n != 2 else [1, -1, 1]
        live = [b for b in range(B) if new[b] > 0 and (total[b] or n < 2)]
        total = [0 if new[b] < 0 else total[b] + 1 for b in range(B)]
        x = r.standard_normal((sum(1 for v in new if v > 0), Hq + 2 * Hkv, D)).astype(np.float16)
        o, _, st = s.step(dev(x), i32(new), 128)
        assert list(host(st.kv_len)) == total and host(st.status)[0] == 0
        cache = [host(t) for t in s.cache]
        q, cu, table = so.rotate(x[:, :Hq], host(st.pos), *(host(t) for t in s.rope)), host(st.cu_new), host(s.table)
        for b in live:
            for h in range(Hq):
                k, _ = so.cache_rows(cache[0], cache[2], table[b], total[b], h * Hkv // Hq, False)
                v, _ = so.cache_rows(cache[1], cache[3], table[b], total[b], h * Hkv // Hq, True)
                want, bound = so.attention(q[cu[b]:cu[b + 1], h].astype(np.float64), k, v, total[b] - 1)
                assert (np.abs(host(o)[cu[b]:cu[b + 1], h] - want) <= bound).all()


def test_step_without_pages_does_nothing(agq):
    s = Server(agq, 2, 16, 3, 4, 2, 64)
    x = dev(rng_of(32).standard_normal((70, 8, 64)).astype(np.float16))
    before = [t.clone() for t in s.cache + [s.table, s.ring]]
    st = agq.kv_map(s.kv_len, i32([40, 30]), s.table, 16, s.ring, s.free, 70)
    assert host(st.status)[0] == 2
    q_out = torch.full((70, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    agq.kv_append(x[:, 4:6], x[:, 6:], st.slot, *s.cache, q=x[:, :4], pos=st.pos, rope_cos=s.rope[0], rope_sin=s.rope[1], q_out=q_out)
    o = torch.full((70, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    agq.attn_kv(q_out, st.cu_new, st.kv_len, s.table, *s.cache, 40, 64, o=o)
    agq.attn_packed(x[:, :4], x[:, 4:6], x[:, 6:], st.cu_new, st.cu_new, o=o)
    assert (o == 7.0).all() and (q_out == 7.0).all()
    assert all(torch.equal(a, b) for a, b in zip(before, s.cache + [s.table, s.ring]))


def test_workspaces_refused(agq):
    """too small, strided, on the host"""
    q, k, cu = torch.zeros(5, 2, 64, dtype=torch.float16, device="cuda"), torch.zeros(4000, 2, 64, dtype=torch.float16, device="cuda"), i32([0, 4000])
    need = agq.attn_packed_workspace_bytes(5, 2, 4000, 2, 64, 1)
    cache = [torch.zeros(s, dtype=torch.int8, device="cuda") for s in ((4, 2, 64, 64), (4, 2, 64, 64), (4, 2), (4, 2))]
    need_kv = agq.attn_kv_workspace_bytes(5, 2, 2, 64, 1, 5, 60000)
    assert need > 0 and need_kv > 0
    packed = lambda ws: agq.attn_packed(q, k, k, i32([0, 5]), cu, workspace=ws)
    kv = lambda ws: agq.attn_kv(q, i32([0, 5]), i32([200]), i32([[0, 1, 2, 3]]), *cache, 5, 60000, workspace=ws)
    for call, n in ((packed, need), (kv, need_kv)):
        with pytest.raises(agq.AgqError):
            call(torch.empty(n - 16, dtype=torch.uint8, device="cuda"))
        with pytest.raises(ValueError):
            call(torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2])
        with pytest.raises(ValueError):
            call(torch.empty(n, dtype=torch.uint8))
        assert (call(torch.empty(n, dtype=torch.uint8, device="cuda")) == 0).all()


def test_generation_captured_and_replayed(agq):
    """two steps (the lengths and the ring's state go there and back) in one graph on another stream, replayed with the
    program's own work in between, against the same steps called one by one"""
    r, B, Hq, Hkv, D = rng_of(33), 2, 8, 2, 128
    a, b = Server(agq, B, 16, 60, Hq, Hkv, D, rows=2048), Server(agq, B, 16, 60, Hq, Hkv, D, rows=2048)
    first = dev(r.standard_normal((45, Hq + 2 * Hkv, D)).astype(np.float16))
    for s in (a, b):
        s.step(first, i32([30, 15]), 1024, prompt=True)
    x = torch.zeros(2, Hq + 2 * Hkv, D, dtype=torch.float16, device="cuda")
    new, kv0, free0 = i32([1, 1]), b.kv_len.clone(), b.free.clone()
    spare = agq.KvStep(*(torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B, B + 1, 2, 2, 2, 1)))
    back = agq.KvStep(kv0, *(torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, 2, 2)), free0, spare.status.clone())
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.kv_len, b.free = kv0, free0
        one, _, _ = b.step(x, new, 1024, out=spare)
        b.kv_len, b.free = spare.kv_len, spare.free_state
        two, _, _ = b.step(x, new, 1024, out=back)
    for n in range(5):
        x.copy_(dev(r.standard_normal(tuple(x.shape)).astype(np.float16)))
        want = [a.step(x, new, 1024)[0] for _ in range(2)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(one, want[0]) and torch.equal(two, want[1]), n
        assert torch.equal(kv0, a.kv_len) and torch.equal(free0, a.free) and all(torch.equal(s, t) for s, t in zip(a.cache, b.cache))
        first.mul_(1.0).sum().item()


def test_two_streams_at_once(agq):
    """two calls in flight on two streams, each with a workspace of its own"""
    r = rng_of(34)
    sides = []
    for n in range(2):
        lens = [3000 + 500 * n]
        table, n_pages = make_pages(r, lens, 64)
        cache = [dev(c) for c in random_cache(r, n_pages, 2, 64, 128)]
        q = dev(random_q(r, 1, 8, 128))
        args = (q, i32([0, 1]), i32(lens), i32(table), *cache, 1, 4096)
        ws = torch.empty(agq.attn_kv_workspace_bytes(1, 8, 2, 128, 1, 1, 4096), dtype=torch.uint8, device="cuda")
        sides.append((args, ws, torch.cuda.Stream(), agq.attn_kv(*args), torch.empty_like(q)))
    torch.cuda.synchronize()
    for _ in range(10):
        for args, ws, stream, _, o in sides:
            with torch.cuda.stream(stream):
                agq.attn_kv(*args, o=o, workspace=ws)
    torch.cuda.synchronize()
    for _, _, _, want, o in sides:
        assert torch.equal(o, want)


# ------------------------------------------------------------------ the softmax's sum and the values' scales

def check_far(agq, q, cu_q, lens, table, cache, max_kv, max_q=1):
    """as check_cache, the scores' bound with what K's form in the matrix instructions adds: sums 128 steps of its page times |q|_1 in size"""
    D, page, Hkv = q.shape[2], cache[0].shape[2], cache[0].shape[1]
    group = q.shape[1] // Hkv
    got = host(agq.attn_kv(dev(q), i32(cu_q), i32(lens), i32(table), *(dev(c) for c in cache), max_q, max_kv)).astype(np.float64)
    for b, L in enumerate(lens):
        step = 2.0 ** cache[2][table[b, :-(-L // page)]].astype(np.float64).max(0)
        for h in range(Hkv):
            k, there = so.cache_rows(cache[0], cache[2], table[b], L, h, False)
            v, _ = so.cache_rows(cache[1], cache[3], table[b], L, h, True)
            for hh in range(h * group, (h + 1) * group):
                x = q[cu_q[b]:cu_q[b + 1], hh].astype(np.float64)
                want, bound = so.attention(x, k, v, L - len(x), True, None, there, offset=128 * step[h] * np.abs(x).sum(-1))
                off = np.abs(got[cu_q[b]:cu_q[b + 1], hh] - want)
                assert np.isfinite(want).all() and (off <= bound).all(), (b, hh, off.max(), np.abs(want).max(), (off - bound).max())


@pytest.mark.parametrize("D,Hq,Hkv,page,n", [(64, 2, 1, 16, 1), (128, 4, 2, 32, 1), (128, 20, 1, 16, 1), (64, 3, 1, 64, 7)])
@pytest.mark.parametrize("lens,loud,max_kv", [([32], [1], 32), ([64], [2], 64), ([1024, 70], [0, 1], 1024), ([2048], [9], 2048), ([16384], [0], 1),
                                              ([16384], [70], 16384), ([30000], [100], 200000)])
@pytest.mark.parametrize("lower", [-2.0, 0.5, 1.0, 3.0, 10.5])
def test_cache_sum_counts_keys_whose_values_are_small(agq, D, Hq, Hkv, page, n, lens, loud, max_kv, lower):
    """pages of zeros, as agq_kv_append writes them (the exponent -30), beside one page of values near fp16's largest (9): the keys
    of the zeros, `lower` powers of two below the others, add nothing to the product with V and most of the softmax's sum.
    In one workgroup of four or eight wavefronts, and shared by several."""
    r, B = rng_of(40, D, Hq, sum(lens), abs(int(10 * lower))), len(lens)
    table, n_pages = make_pages(r, lens, page)
    k = r.integers(-9, 10, (n_pages, Hkv, page, D)).astype(np.int8)
    v = np.zeros((n_pages, Hkv, D, page), np.int8)
    ke, ve = np.full((n_pages, Hkv), -6, np.int8), np.full((n_pages, Hkv), so.E_ZERO, np.int8)
    k[..., 0] = 0
    q = (r.standard_normal((n * B, Hq, D)) * 0.25).astype(np.float16)
    q[..., 0] = 64.0
    for b, j in enumerate(loud):
        p = table[b, min(j * 16, lens[b] - 1) // page]
        k[p, :, :, 0] = np.rint(lower / (64 * D ** -0.5 * np.log2(np.e)) * 64)
        v[p] = r.integers(64, 128, v[p].shape) * r.choice([-1, 1], (Hkv, D, 1))
        ve[p] = 9
    check_far(agq, q, ramp([n] * B), lens, table, (k, v, ke, ve), max_kv, n)


@pytest.mark.parametrize("seed", range(24))
def test_cache_scales_far_apart_in_a_chunk(agq, seed):
    """value scales from end to end of what agq_kv_append makes, the finest and the coarsest of them in every chunk of 64 keys"""
    r, page, lens = rng_of(41, seed), 16, [200, 64, 700]
    D = [64, 128][seed % 2]
    table, n_pages = make_pages(r, lens, page)
    k, v, ke, ve = random_cache(r, n_pages, 2, page, D)
    ve[:] = r.integers(-30, 9, ve.shape)
    for row in table:
        for j in range(0, (row >= 0).sum(), 4):
            ve[row[j + int(r.integers(0, min(4, (row >= 0).sum() - j)))]] = -30
            ve[row[j + int(r.integers(0, min(4, (row >= 0).sum() - j)))]] = 8
    ke[:] = r.integers(-9, -5, ke.shape)
    check_far(agq, random_q(r, 3, 6, D), ramp([1, 1, 1]), lens, table, (k, v, ke, ve), 700)


def test_cache_sum_from_appended_tokens(agq):
    """the same as a server meets it: tokens whose values are zero, one whose values are large, all through agq_kv_append"""
    r, page, T, Hkv, D = rng_of(42), 16, 300, 2, 128
    x = (r.standard_normal((T, 2 * Hkv, D)) * 0.25).astype(np.float16)
    x[:, Hkv:] = 0
    x[130:140, Hkv:] = (r.uniform(20000, 60000, (10, Hkv, D)) * r.choice([-1, 1], (1, Hkv, D))).astype(np.float16)
    cache = [torch.zeros(s, dtype=torch.int8, device="cuda") for s in ((20, Hkv, page, D), (20, Hkv, D, page), (20, Hkv), (20, Hkv))]
    slot = np.arange(T, dtype=np.int32)
    xd = dev(x)
    agq.kv_append(xd[:, :Hkv], xd[:, Hkv:], i32(slot), *cache)
    cache = [host(c).copy() for c in cache]
    assert cache[3].min() == so.E_ZERO and cache[3].max() == 9
    check_far(agq, random_q(r, 1, 4, D), ramp([1]), [T], np.arange(20, dtype=np.int32)[None], cache, T)


# ------------------------------------------------------------------ infinities beside scores that are far apart

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m,at", [(32, 96, 40), (40, 200, 33), (40, 200, 130), (200, 200, 60), (200, 230, 199), (130, 300, 299), (20, 3000, 2000)])
def test_packed_infinity_under_a_louder_key(agq, D, causal, n, m, at):
    """an infinity and a NaN among the first values, then a key whose score is 180 powers of two above theirs: their weights
    are small, not nothing"""
    r = rng_of(43, D, n, m, at)
    q, k, v = np.full((n, 2, D), 8.0, np.float16), np.zeros((m, 1, D), np.float16), r.standard_normal((m, 1, D)).astype(np.float16)
    k[at] = 2.0
    v[0, 0, 3], v[1, 0, 9], v[2, 0, 20], v[at - 1, 0, 31] = np.inf, np.nan, -np.inf, np.inf
    got = check_packed(agq, q, k, v, ramp([n]), ramp([m]), causal, finite=False)
    sees = np.arange(n) + (m - n if causal else m) >= at
    assert sees.any() and not np.isfinite(got[sees][:, :, [3, 9, 20, 31]]).any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,m,quiet", [(1, 1, 1), (5, 40, 40), (40, 40, 33), (140, 300, 300), (70, 200, 64), (6, 3000, 3000), (6, 3000, 1500), (50, 7, 7)])
def test_packed_scores_of_minus_infinity(agq, D, n, m, quiet):
    """keys whose scores are -infinity weigh nothing; a row that sees no others has no softmax and is NaN, a row that sees no key at
    all is 0"""
    r = rng_of(44, D, n, m)
    q, k, v = random_qkv(r, n, m, 2, 1, D)
    q[..., 0] = 1.0
    k[:quiet, :, 0] = -np.inf
    got = check_packed(agq, q, k, v, ramp([n]), ramp([m]), finite=False)
    keys = np.arange(n) + m - n + 1
    assert np.isnan(got[(keys > 0) & (keys <= quiet)]).all() and (got[keys <= 0] == 0).all() and np.isfinite(got[keys > quiet]).all()


# ------------------------------------------------------------------ scores of many millions

@pytest.mark.parametrize("D,group,page", [(64, 1, 16), (128, 4, 64), (128, 20, 128)])
@pytest.mark.parametrize("L,max_kv", [(40, 40), (700, 700), (3000, 3000), (20000, 200000)])
@pytest.mark.parametrize("top,sign", [(700.0, 0), (8000.0, 0), (60000.0, 0), (8000.0, -1), (60000.0, 1)])
def test_cache_scores_of_many_millions(agq, D, group, page, L, max_kv, top, sign):
    """queries of up to 60000 against codes of every size on pages of one scale: the loudest keys take all, however large the scores are;
    all scores negative, and all positive"""
    r = rng_of(50, D, L, int(top), sign + 1)
    table, n_pages = make_pages(r, [L], page)
    pattern = np.ones(D) if sign else r.choice([-1, 1], D)
    size = np.clip(r.integers(-127, 128, (n_pages, 1, page, 1)), -127 if sign <= 0 else 5, 127 if sign >= 0 else -5)
    k, v = (size * pattern).astype(np.int8), r.integers(-127, 128, (n_pages, 1, D, page)).astype(np.int8)
    ke, ve = np.full((n_pages, 1), 9, np.int8), np.full((n_pages, 1), -7, np.int8)
    q = (r.uniform(0.5, 1.0, (2, group, 1)) * top * pattern).astype(np.float16)
    got = host(agq.attn_kv(dev(q), i32([0, 2]), i32([L]), i32(table), *(dev(c) for c in (k, v, ke, ve)), 2, max_kv)).astype(np.float64)
    codes = size[table[0, :-(-L // page)], 0, :, 0].reshape(-1)
    values, _ = so.cache_rows(v, ve, table[0], L, 0, True)
    for i in range(2):
        seen = codes[:L - 1 + i]
        want = values[:L - 1 + i][seen == seen.max()].mean(0)
        assert np.abs(got[i] - want).max() <= 2.0 ** -10, (i, np.abs(got[i] - want).max())


def loud_rows(r, n, m, D, top, key):
    """q [n, D] and k [m, D] of one sign pattern, so that scores are products of two sizes; keys' sizes are 8 / 1024 of `key` apart at least: far
    more, in scores, than the 2^-16 of them that fp32 sums may be off by, so every row's softmax is one key, or those of one size"""
    sign = r.choice([-1.0, 1.0], D)
    size = r.integers(-128, 128, m) * (key / 128)
    return (r.uniform(0.5, 1.0, (n, 1)) * top * sign).astype(np.float16), (size[:, None] * sign).astype(np.float16), size


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [(5, 40), (130, 130), (300, 500), (20, 3000)])
@pytest.mark.parametrize("top,key", [(700.0, 700.0), (3000.0, 3000.0), (8000.0, 8000.0), (60000.0, 60000.0), (20.0, 60000.0), (40.0, 60000.0), (60000.0, 20.0)])
def test_packed_scores_of_many_millions(agq, D, causal, n, m, top, key):
    """queries and keys of up to 60000: a row's loudest keys take all, however large the scores are"""
    r = rng_of(51, D, n, m, int(top), int(key))
    q, k, size = loud_rows(r, 2 * n, m, D, top, key)
    q, k, v = q.reshape(n, 2, D), k.reshape(m, 1, D), r.uniform(-1, 1, (m, 1, D)).astype(np.float16)
    got = host(agq.attn_packed(dev(q), dev(k), dev(v), i32([0, n]), i32([0, m]), causal=causal)).astype(np.float64)
    for i in range(n):
        seen = size[:m - n + i + 1] if causal else size
        want = v[:len(seen), 0].astype(np.float64)[seen == seen.max()].mean(0)
        assert np.abs(got[i] - want).max() <= 2.0 ** -10, (i, np.abs(got[i] - want).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,m", [(130, 130), (300, 300), (20, 3000)])
def test_packed_loud_rows_beside_others(agq, D, n, m):
    """a few queries a thousand times the others, in the same tiles: every row within its own bound"""
    r = rng_of(52, D, n)
    q, k, v = random_qkv(r, n, m, 2, 1, D)
    q[3::17] *= np.float16(1000.0)
    check_packed(agq, q, k, v, ramp([n]), ramp([m]))


# ------------------------------------------------------------------ the ends of the scales' range

@pytest.mark.parametrize("group", [1, 20])
def test_cache_exponents_and_scale_at_their_ends(agq, group):
    """exponents beyond -64 .. 64 are read as the nearer of the two; scores of 2^118, all of them negative, and masked keys beside scores
    of 2^-120"""
    r, page, D, L = rng_of(53, group), 16, 128, 200
    table, n_pages = make_pages(r, [L], page)
    k, v, ke, ve = random_cache(r, n_pages, 1, page, D)
    q, rest = dev(random_q(r, 3, group, D)), (i32([0, 3]), i32([L]), i32(table))
    call = lambda ke, ve, **kw: host(agq.attn_kv(kw.pop("q", q), *rest, *(dev(c) for c in (kw.pop("k", k), v, ke, ve)), 3, L, **kw))
    for far, near in ((-128, -64), (-65, -64), (65, 64), (127, 64)):
        some = r.random(ke.shape) < 0.5
        for one in (0, 1):
            a, b = ((np.where(some, e, ke).astype(np.int8), ve) if one else (ke, np.where(some, e, ve).astype(np.int8)) for e in (far, near))
            assert np.array_equal(call(*a).view(np.uint16), call(*b).view(np.uint16)), (far, one)
    # codes -5 .. -127 of one sign pattern, the same for all of q
    size = r.integers(-127, -4, (n_pages, 1, page, 1))
    loud = dict(q=dev(np.full((3, group, D), 60000.0, np.float16)), k=np.broadcast_to(size, k.shape).astype(np.int8), scale=2.0 ** 24)
    got = call(np.full_like(ke, 64), np.full_like(ve, -7), **loud).astype(np.float64)
    codes, values = size[table[0], 0, :, 0].reshape(-1), so.cache_rows(v, np.full_like(ve, -7), table[0], L, 0, True)[0]
    for i in range(3):
        seen = codes[:L - 2 + i]
        assert np.abs(got[i] - values[:L - 2 + i][seen == seen.max()].mean(0)).max() <= 2.0 ** -10
    got = call(np.full_like(ke, -64), np.full_like(ve, -7), scale=2.0 ** -60).astype(np.float64)      # no score differs from another
    for i in range(3):
        # fp16 weights of one size: the sum's roundings, and the output's
        assert np.abs(got[i] - values[:L - 2 + i].mean(0)).max() <= 2.0 ** -11


def test_packed_scale_at_its_ends(agq):
    r = rng_of(54)
    q, k, v = random_qkv(r, 50, 90, 2, 1, 64)
    check_packed(agq, q, k, v, ramp([50]), ramp([90]), scale=2.0 ** -60)
    got = host(agq.attn_packed(dev(q), dev(k), dev(v), i32([0, 50]), i32([0, 90]), scale=2.0 ** 24)).astype(np.float64)
    s = np.einsum("ihd,jd->ihj", q.astype(np.float64), k[:, 0].astype(np.float64))
    for i in range(50):
        order = np.sort(s[i, :, :41 + i], -1)
        assert (order[:, -1] - order[:, -2] > 2.0 ** -12).all()      # scores of 2^5: fp32 sums are off by less, 2^12 powers of two apart
        assert np.array_equal(got[i], v[:41 + i, 0].astype(np.float64)[s[i, :, :41 + i].argmax(-1)])


# ------------------------------------------------------------------ calls that a program may make

def test_no_tokens_no_requests(agq):
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")
    cache = [torch.ones(s, dtype=torch.int8, device="cuda") for s in ((4, 2, 16, 64), (4, 2, 64, 16), (4, 2), (4, 2))]
    cos = torch.zeros(8, 32, device="cuda")
    q, k = agq.kv_append(h(0, 2, 64), h(0, 2, 64), i32([]), *cache, q=h(0, 4, 64), pos=i32([]), rope_cos=cos, rope_sin=cos)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64) and all((c == 1).all() for c in cache)
    assert agq.attn_kv(h(0, 4, 64), i32([0, 0]), i32([7]), i32([[0]]), *cache, 0, 7).shape == (0, 4, 64)
    assert agq.attn_packed(h(0, 4, 64), h(5, 2, 64), h(5, 2, 64), i32([0, 0]), i32([0, 5])).shape == (0, 4, 64)
    o = h(3, 4, 64) + 7.0
    agq.attn_kv(h(3, 4, 64), i32([0]), i32([]), i32(np.zeros((0, 1))), *cache, 1, 7, o=o)
    agq.attn_packed(h(3, 4, 64), h(5, 2, 64), h(5, 2, 64), i32([0]), i32([0]), o=o)
    assert (o == 7.0).all()
    assert (agq.attn_packed(h(3, 4, 64), h(0, 2, 64), h(0, 2, 64), i32([0, 3]), i32([0, 0]), o=o) == 0).all()
    assert (agq.attn_kv(h(3, 4, 64), i32([0, 3]), i32([0]), i32([[0]]), *cache, 3, 0, o=o + 7.0) == 0).all()

@pytest.mark.parametrize("past,new", [([3], [1]), ([3, 0], [40, 7])])
def test_append_nan_touches_nothing_else(agq, past, new):
    """a NaN has no part in a page's scale; every other entry's code is as if it were 0"""
    r, Hkv, D, page, n_pages = rng_of(55, len(new)), 2, 64, 16, 9
    slot, _ = random_slots(r, past, new, page, n_pages, 1)
    T = len(slot)
    x = r.standard_normal((T, 2 * Hkv, D)).astype(np.float16)
    odd = r.random(x.shape) < 0.02
    odd[0, :, 7] = True
    cache = random_cache(r, n_pages, Hkv, page, D, lo=-9, hi=-9)
    d = [dev(c) for c in cache]
    xd = dev(np.where(odd, np.float16(np.nan), x))
    agq.kv_append(xd[:, :Hkv], xd[:, Hkv:], i32(slot), *d)
    zero = np.where(odd, np.float16(0), x)
    for half, at, turned in ((slice(0, Hkv), 0, False), (slice(Hkv, 2 * Hkv), 1, True)):
        codes, exps = so.kv_append(zero[:, half], slot, cache[at], cache[2 + at], turned)
        same = np.ones(codes.shape, bool)
        for t, h, i in zip(*np.nonzero(odd[:, half])):
            if slot[t] >= 0:
                same[(slot[t] // page, h, i, slot[t] % page) if turned else (slot[t] // page, h, slot[t] % page, i)] = False
        assert np.array_equal(host(d[2 + at]), exps) and np.array_equal(host(d[at])[same], codes[same])


def test_tokens_a_gigabyte_apart(agq):
    """distances between tokens of 2^30 elements (2^24 for packed keys and values): addresses behind 2^32 bytes"""
    r, D, Hq, Hkv, T, far = rng_of(56), 64, 4, 2, 5, 1 << 30
    buf = torch.zeros(4 * far + 16 * D, dtype=torch.float16, device="cuda")
    apart = lambda heads, at, ld=far: buf.as_strided((T, heads, D), (ld, D, 1), at * D)
    q, k, v = random_qkv(r, T, T, Hq, Hkv, D)
    q_far, k_far, v_far, o_far = apart(Hq, 0), apart(Hkv, Hq), apart(Hkv, Hq + Hkv), apart(Hq, Hq + 2 * Hkv)
    for t, x in ((q_far, q), (k_far, k), (v_far, v)):
        t.copy_(dev(x))
    cos, sin = (dev(t) for t in synth.rope_tables(64, D))
    slot, pos, cu, lens, table = i32(np.arange(16, 16 + T)), i32(np.arange(T)), i32([0, T]), i32([T]), i32([[1]])
    near, there = ([torch.zeros(s, dtype=torch.int8, device="cuda") for s in ((2, Hkv, 16, D), (2, Hkv, D, 16), (2, Hkv), (2, Hkv))] for _ in range(2))
    rest = dict(pos=pos, rope_cos=cos, rope_sin=sin)
    want_q, want_k = agq.kv_append(dev(k), dev(v), slot, *near, q=dev(q), **rest)
    agq.kv_append(k_far, v_far, slot, *there, q=q_far, q_out=o_far, k_out=k_far, **rest)
    assert torch.equal(o_far, want_q) and torch.equal(k_far, want_k) and all(torch.equal(a, b) for a, b in zip(near, there))
    assert torch.equal(agq.attn_kv(q_far, cu, lens, table, *there, T, T, o=o_far), agq.attn_kv(dev(q), cu, lens, table, *near, T, T))
    k_wide, v_wide = (buf.as_strided((T, Hkv, D), (1 << 24, D, 1), 4096 + at * D) for at in (0, Hkv))
    k_wide.copy_(dev(k)), v_wide.copy_(dev(v))
    assert torch.equal(agq.attn_packed(q_far, k_wide, v_wide, cu, cu, o=o_far), agq.attn_packed(dev(q), dev(k), dev(v), cu, cu))


def test_pages_that_requests_share(agq):
    """a prompt's pages in several tables, and one page twice in a table: they are read like any others"""
    r, page = rng_of(57), 16
    lens = [200, 170, 100]
    table, n_pages = make_pages(r, lens, page)
    table[1, :9], table[2, :6] = table[0, :9], table[0, :6]
    table[0, 11] = table[0, 2]
    check_cache(agq, random_q(r, 6, 4, 128), ramp([2, 2, 2]), lens, table, random_cache(r, n_pages, 2, page, 128))


def test_joins_captured_and_replayed(agq):
    """both attentions with shared keys in one graph, on one workspace one after the other; lengths, offsets and keys change between the
    replays, and the program works in between"""
    r, Hq, Hkv, D, page = rng_of(58), 4, 1, 128, 64
    n, m, lens = 40, 3000, [20000, 9000]
    table, n_pages = make_pages(r, lens, page)
    cache = [dev(c) for c in random_cache(r, n_pages, Hkv, page, D)]
    q, k, v = (dev(t) for t in random_qkv(r, n, m, Hq, Hkv, D))
    cu_q, cu_k, cu_1, d_len, d_table = i32([0, 25, n]), i32([0, 1000, m]), i32([0, 1, 2]), i32(lens), i32(table)
    most = 200000                                          # more than the lengths, as a program that captures a step says
    ws = torch.empty(max(agq.attn_packed_workspace_bytes(n, Hq, m, Hkv, D, 2), agq.attn_kv_workspace_bytes(2, Hq, Hkv, D, 2, 1, most)),
                     dtype=torch.uint8, device="cuda")
    assert agq.attn_packed_workspace_bytes(n, Hq, m, Hkv, D, 2) > 0 and agq.attn_kv_workspace_bytes(2, Hq, Hkv, D, 2, 1, most) > 0
    o, a = torch.empty(n, Hq, D, dtype=torch.float16, device="cuda"), torch.empty(2, Hq, D, dtype=torch.float16, device="cuda")

    def both(o, a, ws):
        agq.attn_packed(q, k, v, cu_q, cu_k, o=o, workspace=ws)
        agq.attn_kv(o[:2], cu_1, d_len, d_table, *cache, 1, most, o=a, workspace=ws)
    both(o, a, ws)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        both(o, a, ws)
    for cut, key, x, y in ((25, 1000, 20000, 9000), (0, 0, 0, 9000), (39, 2999, 64, 1), (3, 40, 19999, 8999), (25, 1000, 20000, 9000)):
        cu_q.copy_(i32([0, cut, n])), cu_k.copy_(i32([0, key, m])), d_len.copy_(i32([x, y]))
        k.mul_(1.0625)
        o2, a2 = torch.empty_like(o), torch.empty_like(a)
        both(o2, a2, torch.full_like(ws, 255))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(a, a2), (cut, x)
        q.clone().mul_(2.0).sum().item()


# ------------------------------------------------------------------ parts of wider tensors, in and out

@pytest.mark.parametrize("D,Hq,Hkv", [(64, 6, 2), (128, 4, 4)])
@pytest.mark.parametrize("n,lens,max_kv", [(1, [70, 300], 300), (5, [70, 300], 300), (12, [90, 40], 90), (1, [3000, 40], 3000), (6, [3000, 700], 3000),
                                           (3, [20000], 200000)])
def test_cache_in_and_out_of_wider_tensors(agq, D, Hq, Hkv, n, lens, max_kv):
    """several new tokens, q a part of a projection's output and o a part of a wider tensor, whose other bytes stay; one launch, a join, and
    pieces that the device chooses"""
    r, B = rng_of(45, D, n, sum(lens)), len(lens)
    table, n_pages = make_pages(r, lens, 64)
    cache = [dev(c) for c in random_cache(r, n_pages, Hkv, 64, D)]
    T = n * B + 3
    x, wide = dev(random_q(r, T, Hq + 2 * Hkv, D)), torch.full((T, Hq + 3, D), 7.0, dtype=torch.float16, device="cuda")
    rest = (i32(ramp([n] * B) + 1), i32(lens), i32(table), *cache, n, max_kv)
    want = agq.attn_kv(x[:, :Hq].contiguous(), *rest, o=torch.full((T, Hq, D), 7.0, dtype=torch.float16, device="cuda"))
    check_cache(agq, host(x[:, :Hq].contiguous()), ramp([n] * B) + 1, lens, table, [host(c) for c in cache], max_q=n, max_kv=max_kv)
    assert agq.attn_kv(x[:, :Hq], *rest, o=wide[:, 2:2 + Hq]).data_ptr() == wide[:, 2:].data_ptr()
    assert torch.equal(wide[:, 2:2 + Hq], want) and (wide[:, :2] == 7.0).all() and (wide[:, 2 + Hq:] == 7.0).all()
    assert (wide[0] == 7.0).all() and (wide[-2:] == 7.0).all()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 6, 2), (128, 4, 4)])
@pytest.mark.parametrize("n,m", [([70, 300], [70, 300]), ([1, 130], [2500, 4000]), ([100], [3000])])
def test_packed_out_into_a_wider_tensor(agq, D, Hq, Hkv, n, m):
    """o a part of a wider tensor, whose other bytes stay; with and without a join"""
    r = rng_of(46, D, sum(n))
    q, k, v = (dev(t) for t in random_qkv(r, sum(n) + 2, sum(m), Hq, Hkv, D))
    wide = torch.full((sum(n) + 2, Hq + 3, D), 7.0, dtype=torch.float16, device="cuda")
    cu = (i32(ramp(n) + 1), i32(ramp(m)))
    want = agq.attn_packed(q, k, v, *cu, o=torch.full((sum(n) + 2, Hq, D), 7.0, dtype=torch.float16, device="cuda"))
    agq.attn_packed(q, k, v, *cu, o=wide[:, 1:1 + Hq])
    assert torch.equal(wide[:, 1:1 + Hq], want) and (wide[:, :1] == 7.0).all() and (wide[:, 1 + Hq:] == 7.0).all()
    assert (wide[0] == 7.0).all() and (wide[-1] == 7.0).all()
    check_packed(agq, *(host(t) for t in (q, k, v)), ramp(n) + 1, ramp(m))


# ------------------------------------------------------------------ many sequences, and pieces that the device chooses

@pytest.mark.parametrize("D,Hq,Hkv", [(64, 2, 1), (128, 2, 2)])
def test_packed_a_thousand_sequences(agq, D, Hq, Hkv):
    """sixteen times as many as a wavefront looks at together, empty ones and ones of several tiles among them"""
    r = rng_of(47, D)
    n = r.integers(0, 12, 1000)
    n[[3, 500, 999]] = [200, 0, 140]
    m = n + r.integers(0, 9, 1000)
    check_packed(agq, *random_qkv(r, int(n.sum()), int(m.sum()), Hq, Hkv, D), ramp(n), ramp(m))


@pytest.mark.parametrize("max_kv", [64, 4096])
def test_cache_a_thousand_requests(agq, max_kv):
    """in one launch, and with room for several pieces each, of which few requests have more than one"""
    r, page = rng_of(48), 32
    lens = r.integers(0, 60, 1000)
    lens[[0, 640, 999]] = [700, 1500, 900]
    table, n_pages = make_pages(r, lens, page)
    check_cache(agq, random_q(r, 1000, 2, 64), ramp([1] * 1000), lens, table, random_cache(r, n_pages, 1, page, 64), max_kv=max_kv)


@pytest.mark.parametrize("lens,max_kv", [([20000, 3, 0, 9000], 100000), ([16383, 16384, 16385], 60000), ([30000, 70], 90000), ([0, 0, 8000, 1, 0, 5000, 257, 256], 30000)])
@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 4, 1, 64), (64, 6, 2, 16)])
def test_cache_pieces_that_the_device_chooses(agq, lens, max_kv, D, Hq, Hkv, page):
    """max_kv large enough that a CU has 640 keys or more of it, so that the pieces' size comes from the lengths: the workspace has room for the
    pieces that max_kv over the pieces per request makes, not for 512 keys each"""
    r, B = rng_of(49, sum(lens), D), len(lens)
    assert max_kv * B * Hkv >= 256 * 640 and 2 * B <= 256 // Hkv
    most = 4 * (256 // Hkv) // B if B > 4 else 256 // Hkv
    keys = max(1024, -(-(-(-max_kv // most)) // 256) * 256)
    table, n_pages = make_pages(r, lens, page)
    assert agq.attn_kv_workspace_bytes(B, Hq, Hkv, D, B, 1, max_kv) == -(-max_kv // keys) * B * Hq * (D * 4 + 8)
    check_cache(agq, random_q(r, B, Hq, D), ramp([1] * B), lens, table, random_cache(r, n_pages, Hkv, page, D), max_kv=max_kv)


def test_lengths_lowered_between_steps(agq):
    """a draft's tokens that were not taken: the program lowers the lengths inside the requests' pages, the next step writes over them"""
    r, Hq, Hkv, D, page, B = rng_of(59), 4, 2, 64, 16, 2
    s = Server(agq, B, page, 8, Hq, Hkv, D)
    draw = lambda T: r.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float16)
    s.step(dev(draw(30)), i32([20, 10]), 64)
    before = [host(t).copy() for t in (s.table, s.ring, s.free)]
    s.step(dev(draw(9)), i32([4, 5]), 64)
    s.kv_len = i32([21, 12])                               # three and three of them go
    x = draw(3)
    o, _, st = s.step(dev(x), i32([1, 2]), 64)
    assert host(st.status)[0] == 0 and list(host(st.kv_len)) == [22, 14] and list(host(st.pos)) == [21, 12, 13]
    assert all(np.array_equal(a, host(t)) for a, t in zip(before, (s.table, s.ring, s.free)))
    cache, q, cu = [host(t) for t in s.cache], so.rotate(x[:, :Hq], host(st.pos), *(host(t) for t in s.rope)), host(st.cu_new)
    for b, L in enumerate((22, 14)):
        for h in range(Hq):
            k, _ = so.cache_rows(cache[0], cache[2], before[0][b], L, h * Hkv // Hq, False)
            v, _ = so.cache_rows(cache[1], cache[3], before[0][b], L, h * Hkv // Hq, True)
            want, bound = so.attention(q[cu[b]:cu[b + 1], h].astype(np.float64), k, v, L - (cu[b + 1] - cu[b]))
            assert (np.abs(host(o)[cu[b]:cu[b + 1], h] - want) <= bound).all()
