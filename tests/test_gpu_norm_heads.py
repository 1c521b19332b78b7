"""Queries and keys normalised per head and rotated, alone and on the way into the cache, on the GPU against float64
definitions rounded once (oracle/agq_serve_oracle.py)."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import agq_serve_oracle as so  # noqa: E402
from paper_2312_05693_amd import synth  # noqa: E402
from test_gpu_parity import dev, host  # noqa: E402
from test_gpu_serve import agq, i32, random_cache, random_slots, rng_of  # noqa: E402, F401


def heads(r, T, H, D, big=0.02):
    return (r.standard_normal((T, H, D)) * np.where(r.random((T, H, D)) < big, 20, 1)).astype(np.float16)


def gains(r, H, D, own):
    return (1 + 0.2 * r.standard_normal((H, D) if own else D)).astype(np.float16)


def same(got, want):
    """bit for bit, but for NaNs, which have many, and the signs of zeros: a head with an infinity has 1 / rms = 0, and 0 times
    a number has that number's sign, which depends on whether it is the value before or after the rotation"""
    g, w = host(got) if torch.is_tensor(got) else got, np.asarray(want)
    assert g.shape == w.shape and np.array_equal(np.isnan(g), np.isnan(w))
    ok = ~np.isnan(w) & ((g != 0) | (w != 0))
    assert np.array_equal(g.view(np.uint16)[ok], w.view(np.uint16)[ok])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (12, 12), (32, 8), (5, 1), (40, 40)])
@pytest.mark.parametrize("T", [1, 3, 70])
@pytest.mark.parametrize("own", [False, True])
def test_norm_rope(agq, D, Hq, Hkv, T, own):
    r = rng_of(D, Hq, Hkv, T)
    x = heads(r, T, Hq + Hkv, D)
    q, k, g_q, g_k = x[:, :Hq], x[:, Hq:], gains(r, Hq, D, own), gains(r, Hkv, D, own)
    pos = r.integers(0, 500, T)
    cos, sin = synth.rope_tables(512, D)
    d = dev(x)                                        # q and k side by side, as one projection writes them
    got_q, got_k = agq.qk_norm_rope(d[:, :Hq], d[:, Hq:], dev(g_q), dev(g_k), 1e-6, i32(pos), dev(cos), dev(sin))
    same(got_q, so.norm_rotate(q, g_q, 1e-6, pos, cos, sin))
    same(got_k, so.norm_rotate(k, g_k, 1e-6, pos, cos, sin))


def test_norm_rope_many_tokens(agq):
    r = rng_of(2)
    T, H, D = 3000, 20, 128
    x, g, pos = heads(r, T, H, D), gains(r, H, D, True), r.integers(0, 4000, T)
    cos, sin = synth.rope_tables(4096, D)
    got, _ = agq.qk_norm_rope(dev(x), None, dev(g), None, 1e-5, i32(pos), dev(cos), dev(sin))
    same(got, so.norm_rotate(x, g, 1e-5, pos, cos, sin))


@pytest.mark.parametrize("T,Hq,Hkv,D", [(6000, 30, 10, 64), (3001, 31, 3, 128), (20000, 7, 1, 64), (2500, 40, 40, 128)])
@pytest.mark.parametrize("own", [False, True])
def test_norm_rope_several_heads_to_a_lane(agq, T, Hq, Hkv, D, own):
    """so many tokens that the lanes of a head take two heads and more, which they may not share out evenly"""
    r = rng_of(T, Hq, own)
    x, g_q, g_k = (r.standard_normal((T, Hq + Hkv, D)) * 2).astype(np.float16), gains(r, Hq, D, own), gains(r, Hkv, D, own)
    pos = r.integers(0, 700, T)
    cos, sin = synth.rope_tables(700, D)
    d = dev(x)
    got_q, got_k = agq.qk_norm_rope(d[:, :Hq], d[:, Hq:], dev(g_q), dev(g_k), 1e-6, i32(pos), dev(cos), dev(sin))
    same(got_q, so.norm_rotate(x[:, :Hq], g_q, 1e-6, pos, cos, sin))
    same(got_k, so.norm_rotate(x[:, Hq:], g_k, 1e-6, pos, cos, sin))
    if own:                                           # and without a rotation, in place
        q = d[:, :Hq]
        agq.qk_norm_rope(q, None, dev(g_q), None, 1e-6, q_out=q)
        same(d[:, :Hq].contiguous(), so.norm_rotate(x[:, :Hq], g_q, 1e-6))
        assert np.array_equal(host(d[:, Hq:]), x[:, Hq:])


@pytest.mark.parametrize("what", ["q only", "k only", "norm only", "rotation only", "one gain", "in place", "other rows"])
def test_norm_rope_forms(agq, what):
    r = rng_of(3)
    T, Hq, Hkv, D = 9, 6, 2, 64
    q, k, g_q, g_k = heads(r, T, Hq, D), heads(r, T, Hkv, D), gains(r, Hq, D, False), gains(r, Hkv, D, True)
    pos = r.integers(0, 30, T)
    cos, sin = synth.rope_tables(32, D)
    rope = dict(pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin))
    turn = dict(pos=pos, cos=cos, sin=sin)
    dq, dk, dgq, dgk = dev(q), dev(k), dev(g_q), dev(g_k)
    if what == "q only":
        a, b = agq.qk_norm_rope(dq, None, dgq, eps=1e-6, **rope)
        assert b is None
        same(a, so.norm_rotate(q, g_q, 1e-6, **turn))
    elif what == "k only":
        a, b = agq.qk_norm_rope(None, dk, None, dgk, 1e-6, **rope)
        assert a is None
        same(b, so.norm_rotate(k, g_k, 1e-6, **turn))
    elif what == "norm only":
        a, b = agq.qk_norm_rope(dq, dk, dgq, dgk, 1e-6)
        same(a, so.norm_rotate(q, g_q, 1e-6))
        same(b, so.norm_rotate(k, g_k, 1e-6))
    elif what == "rotation only":
        a, b = agq.qk_norm_rope(dq, dk, **rope)
        same(a, so.rotate(q, pos, cos, sin))
        same(b, so.rotate(k, pos, cos, sin))
    elif what == "one gain":
        a, b = agq.qk_norm_rope(dq, dk, None, dgk, 1e-6, **rope)
        same(a, so.rotate(q, pos, cos, sin))
        same(b, so.norm_rotate(k, g_k, 1e-6, **turn))
    elif what == "in place":
        a, b = agq.qk_norm_rope(dq, dk, dgq, dgk, 1e-6, **rope, q_out=dq, k_out=dk)
        assert a is dq and b is dk
        same(dq, so.norm_rotate(q, g_q, 1e-6, **turn))
        same(dk, so.norm_rotate(k, g_k, 1e-6, **turn))
    else:                                             # into and out of wider tensors; gains with a distance between heads
        wide, out = dev(heads(r, T, Hq + Hkv + 3, D)), torch.full((T, Hq + 5, D), 7.0, dtype=torch.float16, device="cuda")
        wide[:, 2:2 + Hq] = dq
        gw = dev(gains(r, Hkv, 2 * D, True))
        gw[:, :D] = dgk
        agq.qk_norm_rope(wide[:, 2:2 + Hq], dk, dgq, gw[:, :D], 1e-6, **rope, q_out=out[:, 1:1 + Hq], k_out=dk)
        same(out[:, 1:1 + Hq].contiguous(), so.norm_rotate(q, g_q, 1e-6, **turn))
        same(dk, so.norm_rotate(k, g_k, 1e-6, **turn))
        assert (host(out[:, 0]) == 7).all() and (host(out[:, 1 + Hq:]) == 7).all()


def test_norm_rope_values_at_their_ends(agq):
    """zeros, subnormals, the largest values, infinities and NaN, each in heads of its own"""
    r = rng_of(4)
    T, H, D = 4, 7, 128
    x = heads(r, T, H, D)
    x[:, 0] = 0
    x[:, 1] = (x[:, 1] * 2.0 ** -20).astype(np.float16)
    x[:, 2] = np.where(r.random((T, D)) < 0.5, 65504, -65504)
    x[:, 3] = 0
    x[:, 3, 70] = 2.0 ** -24
    x[:, 4, 5] = np.inf
    x[:, 5, 100] = np.nan
    g, pos = gains(r, H, D, True), np.array([0, -5, 31, 1000])
    g[6] = 65504
    cos, sin = synth.rope_tables(32, D)
    for eps in (1e-6, 0.0, 0.5):
        with np.errstate(all="ignore"):
            want = so.norm_rotate(x, g, eps, pos, cos, sin)
        got = agq.qk_norm_rope(dev(x), None, dev(g), None, eps, i32(pos), dev(cos), dev(sin))[0]
        same(got, want)


def check_append(agq, r, T, Hq, Hkv, D, page, slot, pos, n_pages, rope=True, own=False, eps=1e-6):
    x = heads(r, T, Hq + 2 * Hkv, D)
    g_q, g_k = gains(r, Hq, D, own), gains(r, Hkv, D, own)
    k_c, v_c, k_e, v_e = random_cache(r, n_pages, Hkv, page, D)
    cos, sin = synth.rope_tables(max(int(pos.max(initial=0)), 1), D)
    d, xd = [dev(a) for a in (k_c, v_c, k_e, v_e)], dev(x)
    q_out, k_out = (torch.full((T, h, D), 7.0, dtype=torch.float16, device="cuda") for h in (Hq, Hkv))
    tables = dict(pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin)) if rope else {}
    turn = dict(pos=pos, cos=cos, sin=sin) if rope else {}
    got_q, got_k = agq.kv_append_norm(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], i32(slot), *d, dev(g_k), eps, q=xd[:, :Hq] if Hq else None,
                                      g_q=dev(g_q) if Hq else None, q_out=q_out if Hq else None, k_out=k_out, **tables)
    on = ((slot >= 0) & (slot < n_pages * page))[:, None, None]
    want_k = so.norm_rotate(x[:, Hq:Hq + Hkv], g_k, eps, **turn)
    same(got_k, np.where(on, want_k, np.float16(7)))
    if Hq:
        same(got_q, np.where(on, so.norm_rotate(x[:, :Hq], g_q, eps, **turn), np.float16(7)))
    for (codes, exps), (gc, ge), turned in ((so.kv_append(want_k, slot, k_c, k_e, False), (d[0], d[2]), 0),
                                            (so.kv_append(x[:, Hq + Hkv:], slot, v_c, v_e, True), (d[1], d[3]), 1)):
        assert np.array_equal(host(gc), codes), turned
        assert np.array_equal(host(ge), exps), turned


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 12, 12), (128, 8, 2), (128, 3, 1), (64, 0, 5)])
@pytest.mark.parametrize("past,new,pad", [([0], [1], 0), ([5, 0, 130], [1, 1, 1], 2), ([0, 7, 0], [200, 33, 1], 3)])
def test_append_norm(agq, page, D, Hq, Hkv, past, new, pad):
    r = rng_of(page, D, len(past), 1)
    T = sum(new) + pad
    n_pages = sum(-(-(p + n) // page) for p, n in zip(past, new)) + 2
    slot, pos = random_slots(r, past, new, page, n_pages, pad)
    check_append(agq, r, T, Hq, Hkv, D, page, slot, pos, n_pages)


@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("T", [40, 1300])
def test_append_norm_forms(agq, rope, own, T):
    r = rng_of(T, rope, own)
    slot, pos = random_slots(r, [3, 0], [T // 2, T - T // 2], 32, 60, 0)
    check_append(agq, r, T, 16, 16, 128, 32, slot, pos, 60, rope=rope, own=own, eps=1e-5)


@pytest.mark.parametrize("own", [False, True])
def test_append_norm_several_heads_to_a_lane(agq, own):
    r = rng_of(77, own)
    slot, pos = random_slots(r, [0, 40, 3], [2500, 1, 1500], 64, 90, 5)
    check_append(agq, r, 4006, 33, 3, 128, 64, slot, pos, 90, own=own)


def test_append_norm_nan_touches_nothing_else(agq):
    """a NaN in a head of a key: that head of that token is NaN; the page's other tokens and heads are as they would be"""
    r = rng_of(78)
    T, Hkv, D, page, n_pages = 20, 3, 64, 32, 4
    slot, pos = random_slots(r, [0], [T], page, n_pages, 0)
    x, g = heads(r, T, 2 * Hkv, D), gains(r, Hkv, D, False)
    bad = x.copy()
    bad[7, 1, 9] = np.nan
    cos, sin = synth.rope_tables(64, D)
    fresh, got = random_cache(r, n_pages, Hkv, page, D), []
    for a in (x, bad):
        d = [dev(c) for c in fresh]
        _, k = agq.kv_append_norm(dev(a)[:, :Hkv], dev(a)[:, Hkv:], i32(slot), *d, dev(g), 1e-6, pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin))
        got.append([host(t) for t in (k, *d)])
    (k0, kc0, vc0, ke0, ve0), (k1, kc1, vc1, ke1, ve1) = got
    assert np.isnan(k1[7, 1]).all() and np.array_equal(np.delete(k1, 7, 0), np.delete(k0, 7, 0)) and np.array_equal(k1[7, [0, 2]], k0[7, [0, 2]])
    assert np.array_equal(vc0, vc1) and np.array_equal(ve0, ve1) and np.array_equal(kc0[:, [0, 2]], kc1[:, [0, 2]]) and np.array_equal(ke0[:, [0, 2]], ke1[:, [0, 2]])
    rest = np.delete(x[:, 1:2], 7, 0)                  # the others' scale is theirs alone
    want = so.norm_rotate(rest, g, 1e-6, np.delete(pos, 7), cos, sin)
    p = slot[0] // page
    e = so.exponent(np.abs(want.astype(np.float64)).max())
    assert ke1[p, 1] == e
    codes = np.clip(np.rint(want[:, 0].astype(np.float64) * 2.0 ** -e), -128, 127)
    assert np.array_equal(np.delete(kc1[p, 1, :T], 7, 0), codes)


def test_append_norm_is_norm_then_append(agq):
    """the cache that the two calls one after the other make"""
    r = rng_of(7)
    T, Hq, Hkv, D, page, n_pages = 50, 8, 4, 64, 16, 12
    x, g_q, g_k = heads(r, T, Hq + 2 * Hkv, D), gains(r, Hq, D, False), gains(r, Hkv, D, False)
    slot, pos = random_slots(r, [0, 9], [30, 20], page, n_pages, 0)
    cos, sin = synth.rope_tables(64, D)
    one, two = ([dev(a) for a in random_cache(rng_of(8), n_pages, Hkv, page, D)] for _ in range(2))
    xd = dev(x)
    q, k, v = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
    rope = dict(pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin))
    q1, k1 = agq.kv_append_norm(k, v, i32(slot), *one, dev(g_k), 1e-6, q=q, g_q=dev(g_q), **rope)
    q2, k2 = agq.qk_norm_rope(q, k, dev(g_q), dev(g_k), 1e-6, **rope)
    agq.kv_append(k2, v, i32(slot), *two)
    assert torch.equal(q1, q2) and torch.equal(k1, k2) and all(torch.equal(a, b) for a, b in zip(one, two))


def test_norm_captured_and_replayed(agq):
    r = rng_of(9)
    T, Hq, Hkv, D, page, n_pages = 8, 8, 2, 128, 16, 10
    slot, pos = random_slots(r, [5] * T, [1] * T, page, n_pages, 0)
    g_q, g_k = dev(gains(r, Hq, D, False)), dev(gains(r, Hkv, D, False))
    cos, sin = (dev(t) for t in synth.rope_tables(64, D))
    slot, pos = i32(slot), i32(pos)
    xd = dev(heads(r, T, Hq + 2 * Hkv, D))
    q, k, v = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
    fresh = random_cache(rng_of(10), n_pages, Hkv, page, D)
    cache, other = [dev(a) for a in fresh], [dev(a) for a in fresh]
    qo, ko, qn, kn = (torch.empty(T, h, D, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hq, Hkv))

    def both(c):
        agq.kv_append_norm(k, v, slot, *c, g_k, 1e-6, q=q, g_q=g_q, pos=pos, rope_cos=cos, rope_sin=sin, q_out=qo, k_out=ko)
        agq.qk_norm_rope(q, k, g_q, g_k, 1e-6, pos, cos, sin, q_out=qn, k_out=kn)
    both(other)
    for a, b in zip(other, fresh):
        a.copy_(dev(b))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(cache)
    for n in range(3):
        xd.copy_(dev(heads(r, T, Hq + 2 * Hkv, D)))
        both(other)
        torch.cuda.synchronize()
        want = [t.clone() for t in (qo, ko, qn, kn)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((qo, ko, qn, kn), want)) and torch.equal(qo, qn) and torch.equal(ko, kn)
        assert all(torch.equal(a, b) for a, b in zip(cache, other)), n


def test_norm_rope_as_large_as_it_gets(agq):
    """T * (Hq + Hkv) * D just below 2^35, in place: 4 GB and more between the first token and the last"""
    r = rng_of(50)
    T, H, D = 4095, 65536, 64
    cos, sin = synth.rope_tables(16, D)
    q, k = (torch.zeros(T, H, D, dtype=torch.float16, device="cuda") for _ in range(2))
    g_q, g_k = gains(r, H, D, False), gains(r, H, D, False)
    rows = [0, 1, 2047, 3071, 3500, T - 1]
    x = [heads(r, len(rows), H, D) for _ in range(2)]
    pos = np.arange(T) % 20
    at = torch.tensor(rows, device="cuda")
    q[at], k[at] = dev(x[0]), dev(x[1])
    agq.qk_norm_rope(q, k, dev(g_q), dev(g_k), 1e-6, i32(pos), dev(cos), dev(sin), q_out=q, k_out=k)
    for t, y, g in ((q, x[0], g_q), (k, x[1], g_k)):
        same(t[at], so.norm_rotate(y, g, 1e-6, pos[rows], cos, sin))
        t[at] = 0
        assert not any(bool(part.any()) for part in t.split(256))


def same_bits(got, want):
    """bit for bit, zeros' signs too: what the definition's zeros are where no head has an infinity"""
    g, w = host(got), np.asarray(want)
    assert g.shape == w.shape and not np.isnan(w).any() and np.array_equal(g.view(np.uint16), w.view(np.uint16))


@pytest.mark.parametrize("T", [5, 1500])
@pytest.mark.parametrize("rope", [True, False])
def test_signs_of_zeros(agq, T, rope):
    """values, gains and angles of zero of either sign, alone and in whole heads; results too small for fp16"""
    r = rng_of(T, rope, 60)
    Hq, Hkv, D, page = 9, 3, 64, 32
    x = heads(r, T, Hq + 2 * Hkv, D)
    x[r.random(x.shape) < 0.5] = 0
    x[:, [0, Hq]] = 0
    x[:, [1, Hq + 1]] = (x[:, [1, Hq + 1]] * 2.0 ** -18).astype(np.float16)
    x = np.where(r.random(x.shape) < 0.5, -x, x)
    g_q, g_k = gains(r, Hq, D, True), gains(r, Hkv, D, True)
    for g in (g_q, g_k):
        g[r.random(g.shape) < 0.2] = 0
        g[r.random(g.shape) < 0.2] *= np.float16(2.0 ** -20)
        g[r.random(g.shape) < 0.3] *= -1
    n_pages = T // page + 3
    slot, pos = random_slots(r, [0], [T], page, n_pages, 0)             # the first token is not turned: sines of 0
    cos, sin = synth.rope_tables(T, D)
    tables = dict(pos=i32(pos), rope_cos=dev(cos), rope_sin=dev(sin)) if rope else {}
    turn = dict(pos=pos, cos=cos, sin=sin) if rope else {}
    want_q, want_k = so.norm_rotate(x[:, :Hq], g_q, 1e-6, **turn), so.norm_rotate(x[:, Hq:Hq + Hkv], g_k, 1e-6, **turn)
    assert np.signbit(want_q[want_q == 0]).any() and not np.signbit(want_q[want_q == 0]).all()
    d = dev(x)
    q, k = agq.qk_norm_rope(d[:, :Hq], d[:, Hq:Hq + Hkv], dev(g_q), dev(g_k), 1e-6, **tables)
    same_bits(q, want_q)
    same_bits(k, want_k)
    cache = [dev(a) for a in random_cache(r, n_pages, Hkv, page, D)]
    q, k = agq.kv_append_norm(d[:, Hq:Hq + Hkv], d[:, Hq + Hkv:], i32(slot), *cache, dev(g_k), 1e-6, q=d[:, :Hq], g_q=dev(g_q), **tables)
    same_bits(q, want_q)
    same_bits(k, want_k)
    if rope:                                                            # q turned without a norm, k normalised
        q, k = agq.qk_norm_rope(d[:, :Hq], d[:, Hq:Hq + Hkv], None, dev(g_k), 1e-6, **tables)
        same_bits(q, so.rotate(x[:, :Hq], pos, cos, sin))
        same_bits(k, want_k)
        cache = [dev(a) for a in random_cache(r, n_pages, Hkv, page, D)]
        q, k = agq.kv_append(d[:, Hq:Hq + Hkv], d[:, Hq + Hkv:], i32(slot), *cache, q=d[:, :Hq], **tables)
        same_bits(q, so.rotate(x[:, :Hq], pos, cos, sin))
        same_bits(k, so.rotate(x[:, Hq:Hq + Hkv], pos, cos, sin))
