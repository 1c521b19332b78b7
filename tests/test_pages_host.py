"""Host-side checks, without a GPU, of the calls for shared pages, normalised heads and log probabilities: every refusal of
include/agq.h comes before any HIP call, sizes are right, the binding refuses tensors that are not what it says, and the
definitions that the GPU tests compare with hold against plain torch."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_serve_host import EINVAL, ESIZE, P, agq, bad_caches, cache_of, tensors  # noqa: E402, F401

Q = P + (1 << 24)         # another plausible address, far from the first


def test_append_norm_refuses(agq):
    ok = dict(cache=cache_of(), k=P, ldk=256, v=P, ldv=256, T=5, slot=P, q=P, ldq=512, Hq=4, g_q=P, ldgq=0, g_k=P, ldgk=0, eps=1e-6, pos=P, cos=P,
              sin=P, rows=64, q_out=P, ldqo=512, k_out=P, ldko=256, stream=None)
    call = lambda **kw: agq.lib().agq_kv_append_norm(*dict(ok, **kw).values())
    for c in bad_caches():
        assert call(cache=c) == EINVAL
    for kw in (dict(k=None), dict(v=None), dict(k=P + 2), dict(ldk=248), dict(ldv=260), dict(T=-1), dict(T=1 << 30), dict(slot=None), dict(ldq=504),
               dict(Hq=0), dict(q=None), dict(q_out=None), dict(ldqo=256), dict(k_out=P + 2), dict(cos=None), dict(pos=None), dict(rows=0),
               dict(g_k=None), dict(g_q=None), dict(g_k=P + 8), dict(g_q=P + 2), dict(ldgq=64), dict(ldgk=132), dict(ldgk=-128), dict(eps=-1e-9),
               dict(eps=float("nan")), dict(q=None, q_out=None, Hq=0)):
        assert call(**kw) == EINVAL, kw
    assert call(T=0) == 0 and call(T=0, k=None, v=None, q=None, g_q=None, g_k=None, slot=None) == 0


def test_qk_norm_rope_refuses(agq):
    ok = dict(q=P, ldq=512, Hq=4, k=P, ldk=256, Hkv=2, T=5, D=128, g_q=P, ldgq=0, g_k=P, ldgk=128, eps=1e-6, pos=P, cos=P, sin=P, rows=64, q_out=P, ldqo=512,
              k_out=P, ldko=256, stream=None)
    call = lambda **kw: agq.lib().agq_qk_norm_rope(*dict(ok, **kw).values())
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(Hq=0), dict(Hkv=0), dict(Hq=-1), dict(Hq=65537), dict(T=-1),
               dict(T=1 << 30), dict(D=96), dict(D=256), dict(q=P + 8), dict(k=P + 2), dict(ldq=504), dict(ldq=516), dict(ldk=128), dict(ldqo=256),
               dict(ldko=250), dict(q_out=P + 4), dict(g_q=P + 8), dict(ldgq=64), dict(ldgk=130), dict(eps=-1.0), dict(eps=float("nan")),
               dict(pos=None), dict(cos=None), dict(sin=None), dict(cos=P + 4), dict(rows=0), dict(pos=P + 2),
               dict(g_q=None, g_k=None, pos=None, cos=None, sin=None),
               dict(q=None, q_out=None, Hq=0), dict(k=None, k_out=None, Hkv=0),
               dict(q=None, q_out=None, Hq=0, g_q=None, k=None, k_out=None, Hkv=0, g_k=None)):
        assert call(**kw) == EINVAL, kw
    assert call(T=0) == 0 and call(T=0, q=None, k=None) == 0


def test_qk_norm_rope_size_limit(agq):
    """T * (Hq + Hkv) * D < 2^35, to the last token; that the largest one below is taken is a test on the GPU"""
    for T, Hq, Hkv, D in ((4096, 65536, 65536, 64), (2048, 65536, 65536, 128), ((1 << 28) + 1, 1, 0, 128), (1 << 28, 1, 1, 64), (613566757, 1, 0, 64),
                          (1 << 22, 100, 100, 64)):
        k = P if Hkv else None
        assert agq.lib().agq_qk_norm_rope(P, Hq * D, Hq, k, max(Hkv, 1) * D, Hkv, T, D, P, 0, k, 0, 1e-6, None, None, None, 0, P, Hq * D, k,
                                          max(Hkv, 1) * D, None) == EINVAL, (T, Hq, Hkv, D)


def far(i):
    return Q + (i << 20)


def pages(**kw):
    return dict(dict(kv_len=far(0), second=far(1), B=3, page=16, table=far(2), max_pages=4, shared=far(3), ring=far(4), n_pages=9, state=far(5)), **kw)


def bad_pages():
    return (dict(B=-1), dict(B=4097), dict(page=0), dict(page=24), dict(page=256), dict(max_pages=0), dict(max_pages=1 << 27), dict(n_pages=0),
            dict(n_pages=1 << 27), dict(kv_len=None), dict(second=None), dict(table=None), dict(shared=None), dict(ring=None), dict(state=None),
            dict(table=far(2) + 2), dict(kv_len_out=None), dict(table_out=None), dict(shared_out=None), dict(state_out=None), dict(status=None),
            dict(kv_len_out=far(0)), dict(kv_len_out=far(0) + 8), dict(kv_len_out=far(0) - 8), dict(table_out=far(2)), dict(table_out=far(2) + 44),
            dict(shared_out=far(3)), dict(shared_out=far(3) - 32), dict(state_out=far(5)), dict(state_out=far(5) + 4))


def test_fork_refuses(agq):
    ok = pages(kv_len_out=far(6), table_out=far(7), shared_out=far(8), src=far(9), dst=far(10), state_out=far(11), status=far(12), stream=None)
    call = lambda **kw: agq.lib().agq_kv_fork(*dict(ok, **kw).values())
    for kw in bad_pages() + (dict(src=None), dict(dst=None), dict(src=far(9) + 1)):
        assert call(**kw) == EINVAL, kw


def test_compact_refuses(agq):
    base = pages()
    ok = dict(kv_len=base["kv_len"], second=base["second"], cu=far(13), keep=far(14), N=7, **{k: base[k] for k in list(base)[2:]}, kv_len_out=far(6),
              table_out=far(7), shared_out=far(8), moves=far(9), state_out=far(11), status=far(12), stream=None)
    call = lambda **kw: agq.lib().agq_kv_compact(*dict(ok, **kw).values())
    for kw in bad_pages() + (dict(cu=None), dict(keep=None), dict(keep=far(14) + 2), dict(N=-1), dict(N=1 << 30), dict(moves=None), dict(moves=far(9) + 8)):
        assert call(**kw) == EINVAL, kw
    f = agq.kv_moves_ints
    assert f(0, 0, 16) > 0 and f(100, 3, 16) - f(0, 0, 16) == 4 * (100 // 16 + 6)
    assert f(-1, 3, 16) == 0 and f(1 << 30, 3, 16) == 0 and f(4, 4097, 16) == 0 and f(4, 4, 17) == 0


def overlaps(outputs, inputs):
    """every output at the start, at the last and just in front of the end of every input and other output: (name, address)"""
    for name, (at, n) in outputs.items():
        for other, (there, m) in {**inputs, **outputs}.items():
            if other != name:
                for place in (there, there + m - 4, there - n + 4):
                    yield name, other, place


def test_fork_refuses_outputs_on_other_tensors(agq):
    """whatever a workgroup writes while another one reads, or both write; addresses that no kernel ever sees"""
    inputs = dict(kv_len=(far(0), 12), second=(far(1), 12), table=(far(2), 48), shared=(far(3), 36), state=(far(5), 8))
    outputs = dict(ring=(far(4), 36), kv_len_out=(far(6), 12), table_out=(far(7), 48), shared_out=(far(8), 36), src=(far(9), 12), dst=(far(10), 12),
                   state_out=(far(11), 8), status=(far(12), 4))
    ok = pages(**{k: outputs[k][0] for k in list(outputs)[1:]}, stream=None)
    for name, other, place in overlaps(outputs, inputs):
        assert agq.lib().agq_kv_fork(*dict(ok, **{name: place}).values()) == EINVAL, (name, other)


def test_compact_refuses_outputs_on_other_tensors(agq):
    moves = 4 * agq.kv_moves_ints(7, 3, 16)
    inputs = dict(kv_len=(far(0), 12), second=(far(1), 12), cu=(far(13), 16), keep=(far(14), 28), table=(far(2), 48), shared=(far(3), 36), state=(far(5), 8))
    outputs = dict(ring=(far(4), 36), kv_len_out=(far(6), 12), table_out=(far(7), 48), shared_out=(far(8), 36), moves=(far(9), moves), state_out=(far(11), 8),
                   status=(far(12), 4))
    base = pages()
    ok = dict(kv_len=base["kv_len"], second=base["second"], cu=far(13), keep=far(14), N=7, **{k: base[k] for k in list(base)[2:]},
              **{k: outputs[k][0] for k in list(outputs)[1:]}, stream=None)
    for name, other, place in overlaps(outputs, inputs):
        assert agq.lib().agq_kv_compact(*dict(ok, **{name: place}).values()) == EINVAL, (name, other)


def test_layers_refuse(agq):
    import ctypes
    two = lambda **kw: (ctypes.c_int64 * 16)(*cache_of(), *cache_of(**kw))
    copy = lambda caches, n=1, src=P, dst=P, m=4: agq.lib().agq_kv_copy_pages(caches, n, src, dst, m, None)
    move = lambda caches, n=1, **kw: agq.lib().agq_kv_move(caches, n, *dict(dict(moves=P, table=P, max_pages=4, stay=P, cu=P, keep=P, N=5, B=2), **kw).values(), None)
    for c in bad_caches():
        assert copy(c) == EINVAL and move(c) == EINVAL
    for kw in (dict(n_pages=9), dict(Hkv=3), dict(D=64), dict(page=32), dict(k=None), dict(v=P + 4)):
        assert copy(two(**kw), 2) == EINVAL and move(two(**kw), 2) == EINVAL, kw
    assert copy(cache_of(), -1) == EINVAL and copy(cache_of(), 65537) == EINVAL and move(cache_of(), -1) == EINVAL
    assert copy(cache_of(), m=-1) == EINVAL and copy(cache_of(), m=(1 << 20) + 1) == EINVAL and copy(cache_of(), src=None) == EINVAL
    assert copy(cache_of(), dst=P + 2) == EINVAL
    assert copy(cache_of(), m=0) == 0 and copy(None, 0) == 0 and copy(cache_of(), m=0, src=None, dst=None) == 0
    for kw in (dict(moves=None), dict(moves=P + 8), dict(table=None), dict(max_pages=0), dict(max_pages=1 << 27), dict(stay=None), dict(cu=None),
               dict(keep=None), dict(N=-1), dict(N=1 << 30), dict(B=-1), dict(B=4097)):
        assert move(cache_of(), **kw) == EINVAL, kw
    assert move(cache_of(), B=0) == 0 and move(None, 0) == 0


def test_logprobs_refuses(agq):
    ok = dict(logits=P, kind=0, T=3, V=100, ld=100, scale=1.0, tokens=P, n_top=4, logprob=P, entropy=P, idx=P, best=P, ws=None, wsb=0, stream=None)
    call = lambda **kw: agq.lib().agq_logprobs(*dict(ok, **kw).values())
    for kw in (dict(logits=None), dict(logits=P + 1), dict(kind=2), dict(kind=-1), dict(kind=1, logits=P + 2), dict(T=-1), dict(T=(1 << 22) + 1), dict(V=0),
               dict(V=(1 << 24) + 1, ld=1 << 25), dict(ld=99), dict(ld=(1 << 30) + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=2.0 ** -25),
               dict(scale=2.0 ** 25), dict(scale=float("nan")), dict(scale=float("inf")), dict(tokens=None), dict(logprob=None), dict(tokens=P + 2),
               dict(logprob=P + 1), dict(entropy=P + 2), dict(n_top=-1), dict(n_top=65), dict(n_top=101), dict(V=3, n_top=4), dict(idx=None), dict(best=None),
               dict(n_top=0), dict(idx=P + 2), dict(best=P + 3)):
        assert call(**kw) == EINVAL, kw
    assert call(T=0) == 0 and call(T=0, logits=None, tokens=None, idx=None) == 0
    g = agq.logprobs_workspace_bytes
    assert g(-1, 100, 0, 4) == 0 and g(1, 0, 0, 0) == 0 and g(1, 100, 2, 0) == 0 and g(1, 100, 0, 65) == 0 and g(0, 100, 0, 0) == 0
    need = g(3, 100000, 0, 4)
    if need:
        assert call(V=100000, ld=100000) == EINVAL and call(V=100000, ld=100000, ws=P + 8, wsb=need) == EINVAL
        assert call(V=100000, ld=100000, ws=P, wsb=need - 1) == ESIZE


def test_logprobs_workspace_sizes(agq):
    """which shapes need a workspace, and that a smaller one is refused for each of them"""
    need = agq.logprobs_workspace_bytes
    for T, V, kind, n_top in ((2, 128000, 0, 20), (40, 70001, 1, 8), (3, 70001, 1, 0), (3, 300001, 0, 0), (600, 600001, 0, 2), (127, 50001, 0, 0)):
        n = need(T, V, kind, n_top)
        assert n > 0 and n % 4 == 0, (T, V, kind, n_top)
        call = lambda ws, size: agq.lib().agq_logprobs(P, kind, T, V, V, 1.0, P, n_top, P, P, P if n_top else None, P if n_top else None, ws, size, None)
        assert call(P, n - 1) == ESIZE and call(P, 0) == ESIZE and call(None, 0) == EINVAL and call(P + 8, n) == EINVAL
    for T, V, kind, n_top in ((600, 2000, 0, 5), (1, 32000, 0, 64), (4096, 32000, 0, 0), (300, 1 << 20, 0, 0), (1, 1, 1, 1), (200, 50001, 1, 8)):
        assert need(T, V, kind, n_top) == 0, (T, V, kind, n_top)


def test_binding_refuses_other_tensors(agq):
    h, i, c = tensors()
    kv = (c(6, 2, 16, 64), c(6, 2, 64, 16), c(6, 2), c(6, 2))
    cos = torch.zeros(8, 32)
    rope = dict(pos=i(3), rope_cos=cos, rope_sin=cos)
    pages = (i(3, 2), 16, i(6), i(6), i(2))
    fork = agq.KvFork(i(3), i(3, 2), i(6), i(3), i(3), i(2), i(1))
    n = agq.kv_moves_ints(5, 3, 16)
    compact = agq.KvCompact(i(3), i(3, 2), i(6), i(n), i(2), i(1))
    layers = agq.kv_layers([kv])
    bad = [lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, None, 1e-6),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(64), 1e-6, q=h(3, 4, 64)),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(64), 1e-6, g_q=h(64)),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(32), 1e-6),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(3, 64), 1e-6),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(64).float(), 1e-6),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(128)[::2], 1e-6),
           lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(64), 1e-6, pos=i(3)),
           lambda: agq.qk_norm_rope(None, None, **rope),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(64), h(64)),
           lambda: agq.qk_norm_rope(h(3, 4, 64), h(2, 2, 64), h(64), h(64)),
           lambda: agq.qk_norm_rope(h(3, 4, 64), h(3, 2, 128), h(64), h(128)),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(2, 64)),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(64), pos=i(3), rope_cos=cos),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(64), pos=i(4), rope_cos=cos, rope_sin=cos),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(64), q_out=h(3, 3, 64)),
           lambda: agq.qk_norm_rope(h(3, 4, 64), None, h(64), k_out=h(3, 4, 64)),
           lambda: agq.qk_norm_rope(h(3, 4, 64).float(), None, h(64)),
           lambda: agq.kv_fork(i(3), i(2), *pages), lambda: agq.kv_fork(i(3).long(), i(3), *pages),
           lambda: agq.kv_fork(i(3), i(3), i(3, 2), 16, i(5), i(6), i(2)), lambda: agq.kv_fork(i(3), i(3), i(3, 4)[:, ::2], 16, i(6), i(6), i(2)),
           lambda: agq.kv_fork(i(3), i(3), *pages, out=fork._replace(copy_src=i(4))),
           lambda: agq.kv_compact(i(3), i(2), i(4), i(5), *pages), lambda: agq.kv_compact(i(3), i(3), i(3), i(5), *pages),
           lambda: agq.kv_compact(i(3), i(3), i(4), i(5).long(), *pages),
           lambda: agq.kv_compact(i(3), i(3), i(4), i(5), *pages, out=compact._replace(moves=i(n - 1))),
           lambda: agq.kv_copy_pages(layers, i(3), i(4)), lambda: agq.kv_copy_pages(layers, i(3).long(), i(3)),
           lambda: agq.kv_move(layers, i(n + 1), i(3, 2), i(3), i(4), i(5)), lambda: agq.kv_move(layers, i(n), i(3, 2), i(3), i(3), i(5)),
           lambda: agq.kv_layers([kv, (c(7, 2, 16, 64), c(7, 2, 64, 16), c(7, 2), c(7, 2))]), lambda: agq.kv_layers([(kv[0], kv[0], kv[2], kv[3])]),
           lambda: agq.logprobs(h(3, 50).double()), lambda: agq.logprobs(h(3, 100)[:, ::2]), lambda: agq.logprobs(h(3, 50).bfloat16()),
           lambda: agq.logprobs(h(3, 50), i(4)), lambda: agq.logprobs(h(3, 50), i(3).long()),
           lambda: agq.logprobs(h(3, 50), out=agq.Logprobs(None, None, None, None)),
           lambda: agq.logprobs(h(3, 50), n_top=2, out=agq.Logprobs(None, torch.zeros(3), None, None)),
           lambda: agq.logprobs(h(3, 50), n_top=2, out=agq.Logprobs(None, torch.zeros(3), i(3, 3), torch.zeros(3, 2))),
           lambda: agq.logprobs(h(3, 50), out=agq.Logprobs(None, torch.zeros(4), None, None))]
    for number, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError("call %d was taken" % number)


def test_binding_refuses_tensors_that_are_not_on_the_gpu(agq):
    """calls that are right but for their device"""
    h, i, c = tensors()
    kv = (c(6, 2, 16, 64), c(6, 2, 64, 16), c(6, 2), c(6, 2))
    cos = torch.zeros(8, 32)
    pages = (i(3, 2), 16, i(6), i(6), i(2))
    layers = agq.kv_layers([kv, kv])
    n = agq.kv_moves_ints(5, 3, 16)
    for call in (lambda: agq.kv_append_norm(h(3, 2, 64), h(3, 2, 64), i(3), *kv, h(64), 1e-6),
                 lambda: agq.qk_norm_rope(h(3, 4, 64), h(3, 2, 64), h(64), h(64), pos=i(3), rope_cos=cos, rope_sin=cos),
                 lambda: agq.kv_fork(i(3), i(3), *pages),
                 lambda: agq.kv_fork(i(3), i(3), *pages, out=agq.KvFork(i(3), i(3, 2), i(6), i(3), i(3), i(2), i(1))),
                 lambda: agq.kv_copy_pages(layers, i(3), i(3)),
                 lambda: agq.kv_compact(i(3), i(3), i(4), i(5), *pages),
                 lambda: agq.kv_move(layers, i(n), i(3, 2), i(3), i(4), i(5)),
                 lambda: agq.logprobs(h(3, 50), i(3), n_top=2),
                 lambda: agq.logprobs(h(3, 50).to("meta"))):
        with pytest.raises(ValueError, match="current GPU"):
            call()


def test_norm_oracle_against_torch():
    from oracle import agq_serve_oracle as so
    g = torch.Generator().manual_seed(3)
    x, gain = torch.randn(5, 3, 64, generator=g).half(), torch.rand(3, 64, generator=g).half()
    want = torch.nn.functional.rms_norm(x.double(), (64,), eps=1e-5) * gain.double()
    assert np.abs(so.norm_rotate(x.numpy(), gain.numpy(), 1e-5).astype(np.float64) - want.numpy()).max() < 2.0 ** -11 * 4
    cos, sin = np.cos(np.arange(7)[:, None] * np.ones(32)).astype(np.float32), np.sin(np.arange(7)[:, None] * np.ones(32)).astype(np.float32)
    turned = so.norm_rotate(x.numpy(), gain.numpy(), 1e-5, np.array([0, 1, 2, 3, 60]), cos, sin).astype(np.float64)
    assert np.array_equal(turned[0], so.norm_rotate(x.numpy(), gain.numpy(), 1e-5)[0])
    ang, w = np.array([1, 2, 3, 6])[:, None, None], want.numpy()[1:]              # the last position is beyond the table
    assert np.abs(turned[1:, :, :32] - (w[..., :32] * np.cos(ang) - w[..., 32:] * np.sin(ang))).max() < 2.0 ** -11 * 4


def test_logprobs_oracle_against_torch():
    from oracle import agq_serve_oracle as so
    g = torch.Generator().manual_seed(4)
    x = torch.randn(6, 90, generator=g, dtype=torch.float64).float() * 3
    x[1, 5:] = -np.inf
    x[2] = -np.inf
    x[3, 7] = np.nan
    x[4, 8] = np.inf
    tokens = [3, 4, 0, 1, 8, 89]
    r = so.logprobs(x.numpy(), tokens, 7, 0.5)
    every = torch.log_softmax(x.double() * 0.5, 1)
    for t in (0, 1, 5):
        assert abs(r["logprob"][t] - every[t, tokens[t]].item()) < 1e-12
        assert abs(r["entropy"][t] - torch.special.entr(every[t].exp()).sum().item()) < 1e-12
        best = torch.sort(x[t].double(), descending=True, stable=True).indices[:7]
        assert r["top_idx"][t].tolist() == best.tolist() and np.allclose(r["top_logprob"][t], every[t, best].numpy(), atol=1e-12)
        assert 0 < r["logprob_bound"][t] < 1e-4 and 0 < r["entropy_bound"][t] < 1e-4
    for t in (2, 3, 4):
        assert np.isnan([r["logprob"][t], r["entropy"][t], *r["top_logprob"][t]]).all() and (r["top_idx"][t] == -1).all()


def test_pages_oracle_by_hand():
    """a fork and a compaction small enough to be followed"""
    from oracle import agq_serve_oracle as so
    table = np.array([[5, 2, -1], [0, -1, -1], [-1, -1, -1]])
    # request 0 has 20 tokens in pages 5 and 2; request 1 has 16 in page 0; free pages 7, 1, 3 from the ring's entry 6 on
    ring, shared = np.array([3, -1, -1, -1, -1, -1, 7, 1]), np.zeros(8, int)
    r = so.kv_fork([20, 16, 0], [0, 0, 0], 16, table, shared, ring, [6, 3], np.full((3, 3), -9))
    lens, out, held, src, dst, ring2, state, status = r
    assert lens == [20, 20, 20] and status == 0 and src == [-1, 2, 2] and dst == [-1, 7, 1]
    assert out.tolist() == [[5, 2, -9], [5, 7, -9], [5, 1, -9]] and held.tolist() == [0, 0, 0, 0, 0, 2, 0, 0]
    assert state == [0, 2] and ring2.tolist() == [3, 0, -1, -1, -1, -1, 7, 1]                # page 0 went back behind page 3
    r = so.kv_compact([20, 20, 20], [20, 3, 17], [0, 0, 2, 2], [10, 19], 16, out, held, ring2, state, np.full((3, 3), -9))
    lens, out2, held2, ring3, state, status, moves = r
    assert lens == [20, 5, 17] and status == 0
    assert moves == [(3, [(5, 0), (5, 1), (5, 2), (5, 10), (7, 3)])]
    assert out2.tolist() == [[5, 2, -9], [3, -9, -9], [5, 1, -9]] and held2.tolist() == [0, 0, 0, 0, 0, 1, 0, 0]
    assert state == [1, 2] and ring3.tolist() == [3, 0, 7, -1, -1, -1, 7, 1]
