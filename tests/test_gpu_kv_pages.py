"""Shared pages, forks and compactions on the GPU against plain definitions, one request, token and page at a time
(oracle/agq_serve_oracle.py): everything bit for bit."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import agq_serve_oracle as so  # noqa: E402
from paper_2312_05693_amd import synth  # noqa: E402
from test_gpu_parity import dev, host  # noqa: E402
from test_gpu_serve import agq, check_cache, i32, random_cache, rng_of  # noqa: E402, F401


class Pool:
    """Requests with pages dealt out at random, some of them held by several (families whose first pages are one), and the ring."""

    def __init__(self, r, lens, page, max_pages, spare, family=1, common=None):
        up = -(-np.asarray(lens, dtype=np.int64) // page)
        B = len(lens)
        common = [0] * B if common is None else common           # pages that request b has from the one before it
        self.n_pages = int((up - np.asarray(common, dtype=np.int64)).sum()) + spare if B else spare
        ids = r.permutation(self.n_pages)
        self.table = r.integers(-5, self.n_pages + 5, (B, max_pages)).astype(np.int32)      # what lies behind is anything
        self.shared = np.zeros(self.n_pages, np.int32)
        at = 0
        for b, u in enumerate(up):
            c = common[b]
            if c:
                self.table[b, :c] = self.table[b - 1, :c]
                self.shared[self.table[b, :c]] += 1
            self.table[b, c:u] = ids[at:at + u - c]
            at += int(u) - c
        self.head = int(r.integers(0, self.n_pages))
        self.ring = np.full(self.n_pages, -1, dtype=np.int32)
        self.ring[(self.head + np.arange(spare)) % self.n_pages] = ids[at:]
        self.state = [self.head, spare]


NAMES = ("kv_len", "block_table", "shared", "copy_src", "copy_dst", "ring", "free_state", "status")


def equal(got, want, names):
    for name, g, w in zip(names, got, want):
        assert np.array_equal(host(g).reshape(-1), np.asarray(w, dtype=np.int64).reshape(-1)), name


def check_fork(agq, pool, lens, parent, page):
    out_table = np.full_like(pool.table, -77)
    want = so.kv_fork(lens, parent, page, pool.table, pool.shared, pool.ring, pool.state, out_table)
    B, max_pages = pool.table.shape
    ring = i32(pool.ring)
    new = lambda *s: torch.full(s, -55, dtype=torch.int32, device="cuda")
    out = agq.KvFork(new(B), i32(out_table), new(pool.n_pages), new(B), new(B), new(2), new(1))
    args = [i32(a) for a in (lens, parent, pool.table)]
    shared, state = i32(pool.shared), i32(pool.state)
    got = agq.kv_fork(*args, page, shared, ring, state, out=out)
    assert got is out
    equal((got.kv_len, got.block_table, got.shared, got.copy_src, got.copy_dst, ring, got.free_state, got.status), want, NAMES)
    for t, a in zip(args + [shared, state], (lens, parent, pool.table, pool.shared, pool.state)):     # inputs stay as they are
        assert np.array_equal(host(t).reshape(-1), np.asarray(a).reshape(-1))
    return want


def families(r, B, width, longest, page):
    """lengths and common pages of families that share the full pages of a prompt"""
    lens, common = np.zeros(B, np.int64), [0] * B
    for f in range(0, B, width):
        prompt = int(r.integers(0, longest + 1))
        for b in range(f, min(B, f + width)):
            lens[b] = prompt + r.integers(0, 2 * page)
            common[b] = prompt // page if b > f else 0
    return lens, common


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("B,width,longest", [(1, 1, 3), (4, 4, 100), (60, 4, 300), (513, 3, 90), (1500, 5, 40), (4096, 8, 20)])
def test_fork(agq, page, B, width, longest):
    r = rng_of(page, B)
    lens, common = families(r, B, width, longest, page)
    most = -(-int(lens.max()) // page) + 1
    pool = Pool(r, lens, page, most, B + 3, common=common)
    parent = np.where(r.random(B) < 0.15, -1, np.minimum(B - 1, np.arange(B) // width * width + r.integers(0, width, B)))
    assert check_fork(agq, pool, lens, parent, page)[-1] == 0


def test_fork_long_requests(agq):
    """rows of many workgroups; pages given back by the thousand, the ring wraps around"""
    r = rng_of(1)
    lens, common = [20000, 20000, 30001, 0, 12000], [0, 700, 0, 0, 0]
    pool = Pool(r, lens, 16, 2000, 1500, common=common)
    assert check_fork(agq, pool, lens, [0, 0, -1, 4, 0], 16)[-1] == 0
    assert check_fork(agq, pool, lens, [-1, -1, -1, -1, -1], 16)[6][1] == pool.n_pages
    assert check_fork(agq, pool, lens, [0, 1, 2, 3, 4], 16)[-1] == 0


@pytest.mark.parametrize("spare", [9000, 40001, 70000])
def test_fork_and_compact_in_large_pools(agq, spare):
    """holders' counts by the ten thousand, pages given back from all over them"""
    r = rng_of(spare)
    lens, common = families(r, 30, 3, 900, 16)
    pool = Pool(r, lens, 16, 70, spare, common=common)
    parent = np.where(r.random(30) < 0.4, -1, np.arange(30) // 3 * 3)
    assert check_fork(agq, pool, lens, parent, 16)[-1] == 0
    stay, kept = losses(r, lens, 16, "all")
    assert check_compact(agq, r, pool, lens, stay, kept, 16, 64, 1)[5] == 0


@pytest.mark.parametrize("what", ["short", "none to spare", "parent", "minus2", "negative", "long", "head", "count"])
def test_fork_leaves_a_step_out(agq, what):
    r = rng_of(2)
    lens, parent = np.array([30, 0, 64, 7]), np.array([0, 0, 2, 0])
    pool = Pool(r, lens, 16, 5, 2)
    if what == "short":
        pool.state[1] = 1
    elif what == "none to spare":
        pool.state[1] = 0
    elif what == "parent":
        parent[1] = 4
    elif what == "minus2":
        parent[3] = -2
    elif what == "negative":
        lens[0] = -3
    elif what == "long":
        lens[2] = 81
    elif what == "head":
        pool.state[0] = -1
    else:
        pool.state[1] = pool.n_pages + 1
    status = check_fork(agq, pool, lens, parent, 16)[-1]
    assert status == {"short": 1, "none to spare": 2}.get(what, -1)


def test_fork_odd_requests(agq):
    """no requests; empty ones; a partly filled page that is shared is copied for all; page numbers outside the cache"""
    r = rng_of(3)
    empty = Pool(r, [], 16, 3, 4)
    assert check_fork(agq, empty, [], [], 16)[-1] == 0
    pool = Pool(r, [0, 0, 0], 16, 3, 4)
    assert check_fork(agq, pool, [0, 0, 0], [2, 2, -1], 16)[-1] == 0
    pool = Pool(r, [20, 32, 20], 16, 3, 9)
    pool.table[2, :2] = pool.table[0, :2]                       # both hold both pages, the second partly filled
    pool.shared[pool.table[0, :2]] = 1
    want = check_fork(agq, pool, [20, 32, 20], [0, 1, 2], 16)
    assert want[4][0] >= 0 and want[4][2] >= 0 and want[4][1] == -1
    check_fork(agq, pool, [20, 32, 20], [2, 2, -1], 16)
    pool = Pool(r, [20, 32, 20], 16, 3, 9)
    pool.table[0, 1], pool.table[1, 0], pool.table[2, 0] = -4, pool.n_pages, 1 << 30
    pool.shared[3] = -8                                         # a count below 0 is taken as 0
    want = check_fork(agq, pool, [20, 32, 20], [0, 0, -1], 16)
    assert want[-1] == 0 and want[3][1] == -4


def test_fork_many_steps(agq):
    """a life of forks, new tokens and ends, each step's outputs the next one's inputs: no page is lost or given twice"""
    r, B, page, n_pages, most = rng_of(5), 12, 16, 200, 20
    lens, table, shared = [0] * B, np.full((B, most), -1, np.int32), np.zeros(n_pages, np.int32)
    ring, state = r.permutation(n_pages).astype(np.int32), [0, n_pages]
    d_ring, d_shared, d_table, d_len, d_state = i32(ring), i32(shared), i32(table), i32(lens), i32(state)
    for n in range(30):
        new = [int(r.integers(1, 40)) if L == 0 and r.random() < 0.4 else 0 if L == 0 or L > 200 else int(r.integers(0, 9)) for L in lens]
        T = sum(new)
        lens, _, _, slot, table, ring, state, status = so.kv_map(lens, new, table, page, ring, state, T)
        step = agq.kv_map(d_len, i32(new), d_table, page, d_ring, d_state, T)
        assert status == 0
        parent = [-1 if r.random() < 0.1 else int(r.integers(0, B)) if r.random() < 0.3 else b for b in range(B)]
        lens, table, shared, src, dst, ring, state, status = so.kv_fork(lens, parent, page, table, shared, ring, state, np.full_like(table, -1))
        out = agq.KvFork(*[torch.full(s, -1, dtype=torch.int32, device="cuda") for s in ((B,), (B, most), (n_pages,), (B,), (B,), (2,), (1,))])
        f = agq.kv_fork(step.kv_len, i32(parent), d_table, page, d_shared, d_ring, step.free_state, out=out)
        equal((f.kv_len, f.block_table, f.shared, f.copy_src, f.copy_dst, d_ring, f.free_state, f.status),
              (lens, table, shared, src, dst, ring, state, status), NAMES)
        assert status == 0
        d_len, d_table, d_shared, d_state = f.kv_len, f.block_table, f.shared, f.free_state
        held = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // page)]]
        free = [int(ring[(state[0] + i) % n_pages]) for i in range(state[1])]
        assert len(set(free)) == len(free) and not set(free) & set(held) and len(set(held)) + len(free) == n_pages
        assert all(held.count(p) == shared[p] + 1 for p in set(held)) and all(shared[p] == 0 for p in free)
    f = agq.kv_fork(d_len, i32([-1] * B), d_table, page, d_shared, d_ring, d_state)
    assert host(f.free_state)[1] == n_pages and not host(f.shared).any()


def check_refused(r, pool, lens, got, ring, copies=()):
    """a step that is left out for its books: copies of the inputs, and the free pages in the ring as they were"""
    head, count = pool.state
    free = (head + np.arange(count)) % pool.n_pages
    assert host(got.status)[0] == -1 and host(got.free_state).tolist() == [head, count]
    assert np.array_equal(host(ring)[free], pool.ring[free])
    assert np.array_equal(host(got.kv_len), lens) and np.array_equal(host(got.shared), pool.shared)
    for t in copies:
        assert (host(t) == -1).all()
    for b, L in enumerate(lens):
        n = -(-int(L) // 16)
        assert np.array_equal(host(got.block_table)[b, :n], pool.table[b, :n])


@pytest.mark.parametrize("spare", [20, 5000, 9000, 40000])            # one launch (one tile of counts, two), three launches
@pytest.mark.parametrize("room", [0, 1, 29])
def test_no_room_in_the_ring(agq, spare, room):
    """free_state says that more pages are free than can be, as 30 pages go back"""
    r = rng_of(spare, room)
    lens = np.array([160, 100, 480, 0, 33])                            # the third one's 30 pages go
    pool = Pool(r, lens, 16, 40, spare)
    pool.state[1] = pool.n_pages - room
    # a ring of other numbers, none of which may change
    pool.ring[:] = r.integers(0, pool.n_pages, pool.n_pages)
    new = lambda *s: torch.full(s, -55, dtype=torch.int32, device="cuda")
    parent = [0, 1, -1, 3, 4]
    B, most = pool.table.shape
    assert so.kv_fork(lens, parent, 16, pool.table, pool.shared, pool.ring, pool.state, pool.table)[-1] == -1
    ring = i32(pool.ring)
    out = agq.KvFork(new(B), new(B, most), new(pool.n_pages), new(B), new(B), new(2), new(1))
    got = agq.kv_fork(i32(lens), i32(parent), i32(pool.table), 16, i32(pool.shared), ring, i32(pool.state), out=out)
    check_refused(r, pool, lens, got, ring, (got.copy_src, got.copy_dst))
    # the same pages, from a request that is cut to nothing; no token moves
    stay, cu, keep = np.array([160, 100, 0, 0, 33]), [0] * 6, np.zeros(0, np.int64)
    assert so.kv_compact(lens, stay, cu, keep, 16, pool.table, pool.shared, pool.ring, pool.state, pool.table)[5] == -1
    ring = i32(pool.ring)
    out = agq.KvCompact(new(B), new(B, most), new(pool.n_pages), new(agq.kv_moves_ints(0, B, 16)), new(2), new(1))
    got = agq.kv_compact(i32(lens), i32(stay), i32(cu), i32(keep), i32(pool.table), 16, i32(pool.shared), ring, i32(pool.state), out=out)
    check_refused(r, pool, lens, got, ring)
    assert host(got.moves)[0] == 0
    # one page of room more than goes back, and exactly as much: taken
    for spare_room in (31, 30):
        pool.state[1] = pool.n_pages - spare_room
        assert check_fork(agq, pool, lens, parent, 16)[-1] == 0


@pytest.mark.parametrize("spare", [6, 8000, 40000])
@pytest.mark.parametrize("room", [0, 2, 4])
def test_no_room_in_the_ring_after_copies(agq, spare, room):
    """pages are taken and given back in the refused step, and the taken ones are free again: the ring's entries that they came from
    are not written over; in one launch with one tile of counts and two, and in three with several"""
    r = rng_of(44, spare)
    lens = np.array([20, 40, 50])
    pool = Pool(r, lens, 16, 5, spare)
    pool.state[1] = pool.n_pages - room
    pool.ring[:] = r.integers(0, pool.n_pages, pool.n_pages)
    new = lambda *s: torch.full(s, -55, dtype=torch.int32, device="cuda")
    for parent in ([0, 0, 0], [-1, 2, 2]):                             # two pages taken, seven given back; one and five
        ring = i32(pool.ring)
        out = agq.KvFork(new(3), new(3, 5), new(pool.n_pages), new(3), new(3), new(2), new(1))
        got = agq.kv_fork(i32(lens), i32(parent), i32(pool.table), 16, i32(pool.shared), ring, i32(pool.state), out=out)
        check_refused(r, pool, lens, got, ring, (got.copy_src, got.copy_dst))
        assert so.kv_fork(lens, parent, 16, pool.table, pool.shared, pool.ring, pool.state, pool.table)[-1] == -1
    pool.state[1] = pool.n_pages - 7
    assert check_fork(agq, pool, lens, [0, 0, 0], 16)[-1] == 0


# ------------------------------------------------------------------ copies

def layers_of(agq, r, n, n_pages, Hkv, page, D, lo=-7, hi=-4):
    caches = [random_cache(r, n_pages, Hkv, page, D, lo, hi) for _ in range(n)]
    d = [tuple(dev(a) for a in c) for c in caches]
    return caches, d, agq.kv_layers(d)


@pytest.mark.parametrize("page,D,Hkv", [(16, 64, 1), (16, 64, 3), (64, 128, 8), (128, 128, 5)])
@pytest.mark.parametrize("layers,n", [(1, 1), (2, 70), (65, 3), (5, 0)])
def test_copy_pages(agq, page, D, Hkv, layers, n):
    r = rng_of(page, Hkv, layers, n)
    n_pages = 2 * n + 5
    caches, d, handle = layers_of(agq, r, layers, n_pages, Hkv, page, D)
    ids = r.permutation(n_pages)
    src, dst = ids[:n].copy(), ids[n:2 * n].copy()
    if n > 2:
        src[1], dst[2] = -1, n_pages                            # left out
        src[0] = src[n - 1]                                     # a page that goes to two places
    agq.kv_copy_pages(handle, i32(src), i32(dst))
    for before, after in zip(caches, d):
        for a, t in zip(before, after):
            a = a.copy()
            for s, e in zip(src, dst):
                if 0 <= s < n_pages and 0 <= e < n_pages:
                    a[e] = a[s]
            assert np.array_equal(host(t), a)


def test_copy_pages_beyond_32_bits(agq):
    """a page whose codes lie more than 4 GB into the cache"""
    n_pages, Hkv, page, D = 70000, 4, 128, 128
    k = torch.empty(n_pages, Hkv, page, D, dtype=torch.int8, device="cuda")
    v = torch.empty(n_pages, Hkv, D, page, dtype=torch.int8, device="cuda")
    e = torch.zeros(n_pages, Hkv, dtype=torch.int8, device="cuda")
    k[69999].random_(-128, 127), v[69999].random_(-128, 127), k[3].random_(-128, 127), v[3].random_(-128, 127)
    e[69999], e[3] = 5, -6
    want = [k[69999].clone(), v[69999].clone(), k[3].clone(), v[3].clone()]
    agq.kv_copy_pages(agq.kv_layers([(k, v, e, e.clone())]), i32([69999, 3]), i32([10, 69998]))
    assert all(torch.equal(a, b) for a, b in zip((k[10], v[10], k[69998], v[69998]), want)) and (e[10] == 5).all() and (e[69998] == -6).all()


# ------------------------------------------------------------------ compactions

def check_compact(agq, r, pool, lens, stay, kept, page, D=64, Hkv=2, layers=1, lo=-7, hi=-4):
    """kept: a list of listed tokens for each request"""
    cu = np.concatenate([[0], np.cumsum([len(k) for k in kept])]).astype(np.int64)
    keep = np.concatenate([np.asarray(k, np.int64) for k in kept] + [np.zeros(0, np.int64)])
    return run_compact(agq, r, pool, lens, stay, cu, keep, page, D, Hkv, layers, lo, hi)


def run_compact(agq, r, pool, lens, stay, cu, keep, page, D=64, Hkv=2, layers=1, lo=-7, hi=-4):
    out_table = np.full_like(pool.table, -77)
    want = so.kv_compact(lens, stay, cu, keep, page, pool.table, pool.shared, pool.ring, pool.state, out_table)
    B, _ = pool.table.shape
    caches, d, handle = layers_of(agq, r, layers, pool.n_pages, Hkv, page, D, lo, hi)
    ring = i32(pool.ring)
    new = lambda *s: torch.full(s, -55, dtype=torch.int32, device="cuda")
    out = agq.KvCompact(new(B), i32(out_table), new(pool.n_pages), new(agq.kv_moves_ints(len(keep), B, page)), new(2), new(1))
    d_stay, d_cu, d_keep, d_table = i32(np.minimum(stay, 2 ** 31 - 1)), i32(cu), i32(keep), i32(pool.table)
    got = agq.kv_compact(i32(lens), d_stay, d_cu, d_keep, d_table, page, i32(pool.shared), ring, i32(pool.state), out=out)
    agq.kv_move(handle, got.moves, d_table, d_stay, d_cu, d_keep)
    equal((got.kv_len, got.block_table, got.shared, ring, got.free_state, got.status), want, ("kv_len", "block_table", "shared", "ring", "free_state", "status"))
    assert np.array_equal(host(d_table), pool.table)
    for before, after in zip(caches, d):
        for i, transposed in ((0, False), (1, True)):
            codes, exps = so.kv_move(before[i], before[2 + i], want[6], transposed)
            assert np.array_equal(host(after[i]), codes) and np.array_equal(host(after[2 + i]), exps)
    return want


def losses(r, lens, page, what):
    stay, kept = [], []
    for b, L in enumerate(lens):
        L = int(L)
        kind = what if what != "all" else ("cut", "drop", "stay", "nothing", "tail", "end")[b % 6]
        s = int(r.integers(0, L + 1))
        some = np.flatnonzero(r.random(L - s) < 0.5) + s
        if kind == "cut":
            some = []
        elif kind == "stay":
            s, some = int(r.choice([L, L + 1, 2 ** 31 - 1])), []
        elif kind == "nothing":
            s, some = 0, []
        elif kind == "tail":                                    # all but a few in the midst
            some = np.arange(min(L, s + int(r.integers(1, page))), L)
        elif kind == "end":
            s = max(0, L - 6)
            some = np.flatnonzero(r.random(L - s) < 0.5) + s
        stay.append(s)
        kept.append(some)
    return stay, kept


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("B,longest,what", [(1, 1, "drop"), (1, 700, "drop"), (7, 400, "all"), (60, 200, "cut"), (70, 100, "all"), (600, 40, "all"),
                                             (1500, 20, "all")])
def test_compact(agq, page, B, longest, what):
    r = rng_of(page, B, longest)
    lens, common = families(r, B, 3, longest, page)
    pool = Pool(r, lens, page, -(-int(lens.max()) // page) + 1, int((lens // page).sum()) + 2 * B + 3, common=common)
    stay, kept = losses(r, lens, page, what)
    assert check_compact(agq, r, pool, lens, stay, kept, page)[5] == 0


@pytest.mark.parametrize("page,D,Hkv,layers", [(16, 128, 1, 3), (64, 128, 8, 2), (128, 64, 5, 1), (32, 64, 12, 66)])
def test_compact_layers_and_scales(agq, page, D, Hkv, layers):
    """exponents far apart: some codes are left with a bit or none"""
    r = rng_of(page, D, Hkv)
    lens = [150, 33, 7, 90]
    pool = Pool(r, lens, page, 11, 40)
    stay, kept = losses(r, lens, page, "drop")
    for lo, hi in ((-128, 127), (-9, -2)):
        assert check_compact(agq, r, pool, lens, stay, kept, page, D, Hkv, layers, lo, hi)[5] == 0


def test_compact_beyond_32_bits(agq):
    """pages whose codes lie more than 4 GB into the cache, old ones and new ones"""
    n_pages, Hkv, page, D = 70000, 4, 128, 128
    k = torch.empty(n_pages, Hkv, page, D, dtype=torch.int8, device="cuda")
    v = torch.empty(n_pages, Hkv, D, page, dtype=torch.int8, device="cuda")
    e = torch.zeros(n_pages, Hkv, dtype=torch.int8, device="cuda")
    r = rng_of(20)
    for p in (69999, 2):
        k[p], v[p] = dev(r.integers(-127, 128, (Hkv, page, D)).astype(np.int8)), dev(r.integers(-127, 128, (Hkv, D, page)).astype(np.int8))
    keep = np.arange(1, 256, 3)
    table, stay, cu, d_keep = i32([[2, 69999]]), i32([1]), i32([0, len(keep)]), i32(keep)
    ring = np.full(n_pages, 5)
    ring[0] = 69998
    c = agq.kv_compact(i32([256]), stay, cu, d_keep, table, page, i32(np.zeros(n_pages)), i32(ring), i32([0, 9]))
    agq.kv_move(agq.kv_layers([(k, v, e, e.clone())]), c.moves, table, stay, cu, d_keep)
    tokens = np.concatenate([[0], keep])
    old_k, old_v = torch.cat([k[2], k[69999]], 1), torch.cat([v[2], v[69999]], 2)
    at = torch.from_numpy(tokens).cuda()
    n = len(tokens)
    assert host(c.status)[0] == 0 and host(c.block_table)[0, 0] == 69998 and host(c.kv_len)[0] == n
    assert torch.equal(k[69998][:, :n], old_k[:, at]) and torch.equal(v[69998][:, :, :n], old_v[:, :, at])
    assert not k[69998][:, n:].any() and not v[69998][:, :, n:].any()


def test_two_streams_at_once(agq):
    """two pools, forked and compacted on streams of their own"""
    jobs = []
    for seed in (1, 2):
        r = rng_of(30, seed)
        lens, common = families(r, 24, 4, 300, 16)
        pool = Pool(r, lens, 16, 24, 400, common=common)
        parent = np.arange(24) // 4 * 4
        caches, d, handle = layers_of(agq, r, 2, pool.n_pages, 4, 16, 128)
        stay, kept = losses(r, lens[parent], 16, "all")
        cu, keep = np.concatenate([[0], np.cumsum([len(k) for k in kept])]), np.concatenate([np.asarray(k, np.int64) for k in kept])
        want = so.kv_fork(lens, parent, 16, pool.table, pool.shared, pool.ring, pool.state, np.full_like(pool.table, -1))
        after = so.kv_compact(want[0], stay, cu, keep, 16, want[1], want[2], want[5], want[6], np.full_like(pool.table, -1))
        assert want[-1] == 0 and after[5] == 0
        codes = []
        for c in caches:
            for i, turned in ((0, False), (1, True)):
                a, b = c[i].copy(), c[2 + i].copy()
                for x, y in zip(want[3], want[4]):
                    if y >= 0:
                        a[y], b[y] = a[x], b[x]
                codes.append(so.kv_move(a, b, after[6], turned))
        jobs.append((pool, d, handle, [i32(x) for x in (lens, parent, pool.table, pool.shared, pool.ring, pool.state, np.minimum(stay, 2 ** 31 - 1), cu, keep)],
                     after, codes))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for i, (s, (pool, d, handle, (lens, parent, table, shared, ring, state, stay, cu, keep), _, _)) in enumerate(zip(streams, jobs)):
        with torch.cuda.stream(s):
            f = agq.kv_fork(lens, parent, table, 16, shared, ring, state)
            agq.kv_copy_pages(handle, f.copy_src, f.copy_dst)
            c = agq.kv_compact(f.kv_len, stay, cu, keep, f.block_table, 16, f.shared, ring, f.free_state)
            agq.kv_move(handle, c.moves, f.block_table, stay, cu, keep)
            got[i] = (f, c)
    torch.cuda.synchronize()
    for (f, c), (pool, d, handle, args, after, codes) in zip(got, jobs):
        equal((c.kv_len, c.shared, args[4], c.free_state, c.status), (after[0], after[2], after[3], after[4], [after[5]]), ("kv_len", "shared", "ring", "free_state", "status"))
        at = 0
        for layer in d:
            for i in (0, 1):
                assert np.array_equal(host(layer[i]), codes[at][0]) and np.array_equal(host(layer[2 + i]), codes[at][1])
                at += 1


def test_compact_long(agq):
    """listed tokens by the ten thousand, pages by the thousand"""
    r = rng_of(11)
    lens = [30000, 3, 17001]
    pool = Pool(r, lens, 16, 2000, 3000)
    stay, kept = losses(r, lens, 16, "drop")
    stay[0], kept[0] = 5, np.arange(5, 30000, 2)
    assert check_compact(agq, r, pool, lens, stay, kept, 16)[5] == 0


def test_compact_shared_last_page(agq):
    """a request that is cut inside a page that another one holds gets its own; one that stays as it is does not"""
    r = rng_of(12)
    lens, common = [64, 64, 50], [0, 4, 0]
    pool = Pool(r, lens, 16, 5, 6, common=common)
    want = check_compact(agq, r, pool, lens, [40, 64, 50], [[], [], []], 16)
    assert len(want[6]) == 1 and want[1][0, 2] != pool.table[0, 2] and want[1][1, 2] == pool.table[1, 2]
    want = check_compact(agq, r, pool, lens, [48, 30, 33], [[], [], []], 16)
    assert len(want[6]) == 1 and want[1][2, 2] == pool.table[2, 2]


@pytest.mark.parametrize("what", ["short", "descends", "twice", "below", "beyond", "sums", "sums beyond", "negative stay", "negative", "long", "head", "count"])
def test_compact_leaves_a_step_out(agq, what):
    r = rng_of(13)
    lens, stay = np.array([40, 20, 64]), np.array([10, 20, 33])
    cu, keep = np.array([0, 4, 4, 9]), np.array([12, 20, 21, 39, 35, 40, 41, 50, 63])
    pool = Pool(r, lens, 16, 4, 8)
    if what == "short":                  # 14 tokens and 33 + 5 are to lie in new pages from entries 0 and 2 on: one each
        pool.state[1] = 0
    elif what == "descends":
        keep[2] = 19
    elif what == "twice":
        keep[6] = 40
    elif what == "below":
        keep[0] = 9
    elif what == "beyond":
        keep[8] = 64
    elif what == "sums":
        cu[2] = 3
    elif what == "sums beyond":
        cu[3] = 10
    elif what == "negative stay":
        stay[1] = -1
    elif what == "negative":
        lens[1] = -1
    elif what == "long":
        lens[1] = 65
    elif what == "head":
        pool.state[0] = pool.n_pages
    else:
        pool.state[1] = -1
    want = run_compact(agq, r, pool, lens, stay, cu, keep, 16)
    assert want[5] == (2 if what == "short" else -1)


@pytest.mark.parametrize("spare", [8, 9000])                        # one launch, three
@pytest.mark.parametrize("cu", [[-3, 4, 4, 9], [-(1 << 31), -5, 4, 9], [0, -1, 4, 9], [-3, -2, -1, -1], [(1 << 31) - 1] * 4])
def test_compact_sums_outside(agq, spare, cu):
    r = rng_of(23)
    lens, stay = np.array([40, 20, 64]), np.array([10, 20, 33])
    pool = Pool(r, lens, 16, 4, spare)
    keep = np.array([12, 20, 21, 39, 35, 40, 41, 50, 63])
    assert run_compact(agq, r, pool, lens, stay, np.array(cu), keep, 16)[5] == -1


def test_compact_odd_requests(agq):
    r = rng_of(14)
    pool = Pool(r, [], 16, 3, 4)
    assert check_compact(agq, r, pool, [], [], [], 16)[5] == 0
    pool = Pool(r, [0, 5], 16, 3, 4)
    assert check_compact(agq, r, pool, [0, 5], [0, 0], [[], [4]], 16)[5] == 0
    # entries of no request, in front of the first and behind the last, are not looked at
    pool = Pool(r, [20, 9], 16, 3, 6)
    assert run_compact(agq, r, pool, [20, 9], [2, 0], np.array([2, 4, 5]), np.array([99, -1, 7, 19, 3, 1 << 30]), 16)[5] == 0
    # a page number outside the cache: its tokens are 0, and no other memory is touched
    pool = Pool(r, [40, 9], 16, 4, 6)
    caches, d, handle = layers_of(agq, r, 1, pool.n_pages, 2, 16, 64)
    pool.table[0, 1] = -3
    t, stay, cu, keep = i32(pool.table), i32([3, 9]), i32([0, 3, 3]), i32([5, 20, 35])
    got = agq.kv_compact(i32([40, 9]), stay, cu, keep, t, 16, i32(pool.shared), i32(pool.ring), i32(pool.state))
    agq.kv_move(handle, got.moves, t, stay, cu, keep)
    new = int(host(got.block_table)[0, 0])
    assert host(got.status)[0] == 0 and new == pool.ring[pool.head]
    k = host(d[0][0])
    assert not k[new, :, 4].any() and np.array_equal(np.delete(k, new, 0), np.delete(caches[0][0], new, 0))


@pytest.mark.parametrize("spare", [120, 9000])
def test_captured_and_replayed(agq, spare):
    """a fork and a compaction in one graph, replayed with other lengths and parents, against eager calls"""
    r, B, page, most = rng_of(15), 16, 16, 12
    lens, common = families(r, B, 4, 100, page)
    pool = Pool(r, lens, page, most, spare, common=common)
    caches, d, handle = layers_of(agq, r, 3, pool.n_pages, 4, page, 64)
    _, d2, handle2 = layers_of(agq, r, 3, pool.n_pages, 4, page, 64)
    N = 40
    d_len, parent, table, shared, state = i32(lens), i32(np.arange(B)), i32(pool.table), i32(pool.shared), i32(pool.state)
    stay, cu, keep = i32(np.zeros(B)), i32(np.zeros(B + 1)), i32(np.zeros(N))

    def outs():
        new = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        return (agq.KvFork(new(B), new(B, most), new(pool.n_pages), new(B), new(B), new(2), new(1)),
                agq.KvCompact(new(B), new(B, most), new(pool.n_pages), new(agq.kv_moves_ints(N, B, page)), new(2), new(1)))

    def both(ring, h, fo, co):
        f = agq.kv_fork(d_len, parent, table, page, shared, ring, state, out=fo)
        agq.kv_copy_pages(h, f.copy_src, f.copy_dst)
        c = agq.kv_compact(f.kv_len, stay, cu, keep, f.block_table, page, f.shared, ring, f.free_state, out=co)
        agq.kv_move(h, c.moves, f.block_table, stay, cu, keep)
    rings = [i32(pool.ring), i32(pool.ring)]
    o1, o2 = outs(), outs()
    both(rings[0], handle, *o1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(rings[0], handle, *o1)
    for n in range(4):
        p = np.minimum(B - 1, np.arange(B) // 4 * 4 + r.integers(0, 4, B))
        if n == 2:
            p[:4] = -1
        after = [int(lens[x]) if x >= 0 else 0 for x in p]
        s = [int(r.integers(0, L + 1)) for L in after]
        listed, c = [], [0]
        for L, x in zip(after, s):
            listed += sorted(r.choice(np.arange(x, L), min(2, L - x), replace=False).tolist())
            c.append(len(listed))
        parent.copy_(i32(p)), stay.copy_(i32(s)), cu.copy_(i32(c)), keep.copy_(i32(listed + [0] * (N - len(listed))))
        for ring in rings:
            ring.copy_(i32(pool.ring))
        for a, b in zip(d, d2):
            fresh = random_cache(r, pool.n_pages, 4, page, 64)
            for x, y, z in zip(a, b, fresh):
                x.copy_(dev(z)), y.copy_(dev(z))
        both(rings[1], handle2, *o2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert host(o2[0].status)[0] == 0 and host(o2[1].status)[0] == 0
        L = host(o2[1].kv_len)
        for x, y in zip(o1, o2):
            for name, g, w in zip(x._fields, x, y):
                if name == "block_table":
                    lens_of = host(x.kv_len)
                    for b in range(B):
                        u = -(-int(lens_of[b]) // page)
                        assert np.array_equal(host(g)[b, :u], host(w)[b, :u])
                elif name != "moves":
                    assert torch.equal(g, w), name
        assert torch.equal(rings[0], rings[1]) and L.max() > 0
        for a, b in zip(d, d2):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), n


# ------------------------------------------------------------------ together, as a program uses them

@pytest.mark.parametrize("D,Hq,Hkv,page", [(64, 4, 2, 16), (128, 8, 8, 32)])
def test_beams(agq, D, Hq, Hkv, page):
    """Prompts, then a beam search: scores of the logits, forks by the best continuations, normalised heads into the pages and
    attention over them, and tokens pruned on the way.  A mirror of every request's keys and values, as the cache is to hold
    them, goes through the same forks and losses on the host; the attention is compared with it after every step."""
    r, W, prompts, V, eps = rng_of(D, page, 31), 3, 2, 500, 1e-6
    B, most = W * prompts, 10
    lens0 = [37, 20]
    n_pages = 80
    caches, d, handle = layers_of(agq, r, 2, n_pages, Hkv, page, D)
    table, shared, ring, state = i32(np.full((B, most), -1)), i32(np.zeros(n_pages)), i32(r.permutation(n_pages)), i32([0, n_pages])
    kv_len = i32([0] * B)
    cos, sin = synth.rope_tables(256, D)
    dc, ds = dev(cos), dev(sin)
    g_q, g_k = (1 + 0.2 * r.standard_normal(D)).astype(np.float16), (1 + 0.2 * r.standard_normal(D)).astype(np.float16)
    dgq, dgk = dev(g_q), dev(g_k)
    mirror = [[(d[l][0].cpu().numpy().copy(), d[l][1].cpu().numpy().copy(), d[l][2].cpu().numpy().copy(), d[l][3].cpu().numpy().copy())] for l in range(2)]
    host_table, lens, offset = np.full((B, most), -1, np.int32), [0] * B, np.zeros(B, np.int64)
    h_shared, h_ring, h_state = np.zeros(n_pages, np.int32), host(ring).copy(), [0, n_pages]
    score = np.zeros(B)

    def step(new):
        nonlocal kv_len, state, lens, host_table, h_ring, h_state
        T = sum(new)
        before = list(lens)
        m = agq.kv_map(kv_len, i32(new), table, page, ring, state, T)
        lens, cu, pos, slot, host_table, h_ring, h_state, status = so.kv_map(lens, new, host_table, page, h_ring, h_state, T)
        assert status == 0 and host(m.status)[0] == 0 and np.array_equal(host(m.slot), slot)
        kv_len, state = m.kv_len, m.free_state
        where = np.concatenate([before[b] + offset[b] + np.arange(n) for b, n in enumerate(new)]).astype(np.int32)
        x = r.standard_normal((T, Hq + 2 * Hkv, D)).astype(np.float16)
        xd = dev(x)
        for l in range(2):
            q, k = agq.kv_append_norm(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], m.slot, *d[l], dgk, eps, q=xd[:, :Hq], g_q=dgq, pos=i32(where),
                                      rope_cos=dc, rope_sin=ds)
            kc, vc, ke, ve = mirror[l][0]
            want_k = so.norm_rotate(x[:, Hq:Hq + Hkv], g_k, eps, where, cos, sin)
            kc, ke = so.kv_append(want_k, slot, kc, ke, False)
            vc, ve = so.kv_append(x[:, Hq + Hkv:], slot, vc, ve, True)
            mirror[l][0] = (kc, vc, ke, ve)
        o = agq.attn_kv(q, m.cu_new, m.kv_len, table, *d[1], max_q=max(new), max_kv=max(lens))
        # against float64 attention over what the host holds
        qh, got, cuh = host(q).astype(np.float64), host(o).astype(np.float64), np.asarray(cu)
        kc, vc, ke, ve = mirror[1][0]
        for b in range(B):
            if new[b] <= 0:
                continue
            for h in range(Hq):
                keys, _ = so.cache_rows(kc, ke, host_table[b], lens[b], h // (Hq // Hkv), False)
                vals, _ = so.cache_rows(vc, ve, host_table[b], lens[b], h // (Hq // Hkv), True)
                qq = qh[cuh[b]:cuh[b + 1], h]
                offs = 128 * 2.0 ** ke[host_table[b, :-(-lens[b] // page)], h // (Hq // Hkv)].astype(np.float64).max() * np.abs(qq).sum(1)
                w, bound = so.attention(qq, keys, vals, lens[b] - new[b], offset=offs)
                assert (np.abs(got[cuh[b]:cuh[b + 1], h] - w) <= bound).all()

    def same_caches():
        for l in range(2):
            for g, w in zip(d[l], mirror[l][0]):
                assert np.array_equal(host(g), w)

    step([lens0[b // W] if b % W == 0 else 0 for b in range(B)])
    parent = np.array([b // W * W for b in range(B)])
    for n in range(6):
        f = agq.kv_fork(kv_len, i32(parent), table, page, shared, ring, state)
        agq.kv_copy_pages(handle, f.copy_src, f.copy_dst)
        lens, host_table, h_shared, src, dst, h_ring, h_state, status = so.kv_fork(lens, parent, page, host_table, h_shared, h_ring, h_state, host_table)
        assert status == 0 and host(f.status)[0] == 0
        for l in range(2):
            parts = tuple(a.copy() for a in mirror[l][0])
            for s, e in zip(src, dst):
                if e >= 0:
                    for a in parts:
                        a[e] = a[s]
            mirror[l][0] = parts
        same_caches()
        kv_len, table, shared, state = f.kv_len, f.block_table, f.shared, f.free_state
        offset = offset[parent]
        step([1] * B)
        logits = (r.standard_normal((B, V)) * 2).astype(np.float16)
        best = agq.logprobs(dev(logits), n_top=W)
        want = so.logprobs(logits, None, W)
        assert np.array_equal(host(best.top_idx), want["top_idx"])
        total = score[:, None] + host(best.top_logprob)
        parent = np.concatenate([np.sort(p * W + np.argsort(-total[p * W:(p + 1) * W].reshape(-1), kind="stable")[:W] // W) for p in range(prompts)])
        score = total.max(1)[parent]
        if n == 3:                                              # every other token behind the first four goes
            stay, kept = [4] * B, [np.arange(4, L, 2) for L in lens]
            cu = np.concatenate([[0], np.cumsum([len(k) for k in kept])])
            keep = np.concatenate(kept)
            before = np.array(lens)
            args = i32(stay), i32(cu), i32(keep)
            c = agq.kv_compact(kv_len, *args, table, page, shared, ring, state)
            agq.kv_move(handle, c.moves, table, *args)
            lens, host_table, h_shared, h_ring, h_state, status, moves = so.kv_compact(lens, stay, cu, keep, page, host_table, h_shared, h_ring, h_state,
                                                                                       host_table)
            assert status == 0 and host(c.status)[0] == 0
            for l in range(2):
                kc, vc, ke, ve = mirror[l][0]
                kc, ke = so.kv_move(kc, ke, moves, False)
                vc, ve = so.kv_move(vc, ve, moves, True)
                mirror[l][0] = (kc, vc, ke, ve)
            same_caches()
            kv_len, table, shared, state = c.kv_len, c.block_table, c.shared, c.free_state
            offset = offset + before - np.array(lens)
            h_state = list(h_state)
    end = agq.kv_fork(kv_len, i32([-1] * B), table, page, shared, ring, state)
    assert host(end.free_state)[1] == n_pages and not host(end.shared).any()
