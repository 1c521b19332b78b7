"""Host-side checks of the serving calls, without a GPU: every refusal of include/agq.h comes before any HIP call, sizes
are right, and the binding refuses tensors that are not what it says."""
from __future__ import annotations

import ctypes

import pytest

torch = pytest.importorskip("torch")

EINVAL, ESIZE = -1, -2
P = 1 << 20          # plausible, aligned, never dereferenced: every call below fails its checks or does nothing


@pytest.fixture(scope="module")
def agq():
    from paper_2312_05693_amd import build
    build.build(force=False)
    from paper_2312_05693_amd import binding
    binding.lib()
    return binding


def cache_of(k=P, v=P, ke=P, ve=P, n_pages=8, Hkv=2, D=128, page=16):
    return (ctypes.c_int64 * 8)(k or 0, v or 0, ke or 0, ve or 0, n_pages, Hkv, D, page)


def bad_caches():
    for kw in (dict(k=None), dict(v=None), dict(ke=None), dict(ve=None), dict(k=P + 8), dict(v=P + 4), dict(n_pages=0), dict(n_pages=1 << 28),
               dict(Hkv=0), dict(D=96), dict(D=256), dict(page=8), dict(page=48), dict(page=256), dict(page=0)):
        yield cache_of(**kw)
    yield None


def test_map_refuses(agq):
    ok = dict(kv_len=P, n_new=P + 4096, B=3, page=16, table=P, max_pages=4, ring=P, n_pages=9, state=P, T=3, kv_len_out=P + 64, cu=P, pos=P, slot=P,
              state_out=P + 8, status=P, stream=None)
    call = lambda **kw: agq.lib().agq_kv_map(*dict(ok, **kw).values())
    for kw in (dict(B=-1), dict(B=(1 << 20) + 1), dict(T=-1), dict(T=1 << 31), dict(page=0), dict(page=24), dict(page=256), dict(max_pages=0),
               dict(max_pages=1 << 27), dict(n_pages=0), dict(n_pages=1 << 27), dict(kv_len=None), dict(n_new=None), dict(table=None), dict(ring=None),
               dict(state=None), dict(kv_len_out=None), dict(cu=None), dict(pos=None), dict(slot=None), dict(state_out=None), dict(status=None),
               dict(table=P + 2), dict(kv_len_out=P), dict(kv_len_out=P + 8), dict(kv_len_out=P - 8), dict(state_out=P), dict(state_out=P + 4)):
        assert call(**kw) == EINVAL, kw


def test_append_refuses(agq):
    ok = dict(cache=cache_of(), k=P, ldk=256, v=P, ldv=256, T=5, slot=P, q=P, ldq=512, Hq=4, pos=P, cos=P, sin=P, rows=64, q_out=P, ldqo=512, k_out=P,
              ldko=256, stream=None)
    call = lambda **kw: agq.lib().agq_kv_append(*dict(ok, **kw).values())
    for c in bad_caches():
        assert call(cache=c) == EINVAL
    for kw in (dict(k=None), dict(v=None), dict(k=P + 2), dict(v=P + 8), dict(ldk=248), dict(ldk=260), dict(ldv=128), dict(T=-1), dict(T=1 << 30),
               dict(slot=None), dict(slot=P + 1), dict(ldq=504), dict(ldq=516), dict(Hq=0), dict(Hq=-4), dict(q=None), dict(q_out=None), dict(q=P + 4),
               dict(q_out=P + 8), dict(ldqo=256), dict(k_out=P + 2), dict(ldko=250), dict(cos=None), dict(sin=None), dict(pos=None), dict(rows=0),
               dict(cos=P + 4), dict(cos=None, sin=None, pos=None), dict(cos=None, sin=None, pos=None, q=None, q_out=None, Hq=0)):
        assert call(**kw) == EINVAL, kw
    assert call(T=0) == 0
    assert call(T=0, q=None, q_out=None, Hq=0, k_out=None, cos=None, sin=None, pos=None) == 0


def test_packed_refuses(agq):
    ok = dict(q=P, ldq=512, Tq=5, Hq=4, k=P, ldk=256, v=P, ldv=256, Tk=7, Hkv=2, D=128, cu_q=P, cu_k=P, B=2, causal=1, scale=0.1, o=P, ldo=512, ws=None, wsb=0,
              stream=None)
    call = lambda **kw: agq.lib().agq_attn_packed(*dict(ok, **kw).values())
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=P + 8), dict(k=P + 8), dict(v=P + 2), dict(o=P + 4), dict(ldq=511),
               dict(ldq=504), dict(ldk=128), dict(ldv=260), dict(ldo=500), dict(Tq=-1), dict(Tk=-1), dict(Tq=1 << 31), dict(Hq=3), dict(Hq=0), dict(Hkv=0),
               dict(Hq=1), dict(D=32), dict(D=80), dict(D=256), dict(cu_q=None), dict(cu_k=None), dict(cu_q=P + 2), dict(B=-1), dict(B=1 << 21),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(Tq=1 << 30, Hq=1024, Hkv=1024)):
        assert call(**kw) == EINVAL, kw
    assert call(Tq=0) == 0 and call(B=0) == 0
    assert call(ldk=(1 << 24) + 8) == EINVAL and call(ldv=(1 << 24) + 8) == EINVAL
    # few queries and many keys share the keys between workgroups, which takes a workspace
    need = agq.attn_packed_workspace_bytes(5, 4, 9000, 2, 128, 1)
    assert need > 0 and need % (5 * 4 * (128 * 4 + 8)) == 0
    assert call(B=1, Tk=9000) == EINVAL and call(B=1, Tk=9000, ws=P + 4, wsb=need) == EINVAL
    assert call(B=1, Tk=9000, ws=P, wsb=need - 1) == ESIZE


def test_cache_attention_refuses(agq):
    ok = dict(cache=cache_of(), q=P, ldq=512, T=3, Hq=4, cu_q=P, kv_len=P, B=3, table=P, max_pages=4, max_q=1, max_kv=64, scale=0.1, o=P, ldo=512, ws=None,
              wsb=0, stream=None)
    call = lambda **kw: agq.lib().agq_attn_kv(*dict(ok, **kw).values())
    for c in bad_caches():
        assert call(cache=c) == EINVAL
    for kw in (dict(q=None), dict(o=None), dict(q=P + 8), dict(o=P + 2), dict(ldq=504), dict(ldo=520 - 16), dict(ldq=516), dict(T=-1), dict(T=1 << 31),
               dict(Hq=3), dict(Hq=0), dict(Hq=4096, ldq=4096 * 128, ldo=4096 * 128), dict(cu_q=None), dict(kv_len=None), dict(table=None),
               dict(table=P + 2), dict(B=-1), dict(B=65536), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(max_q=-1), dict(max_kv=-1),
               dict(max_kv=(1 << 30) + 1), dict(max_q=(1 << 30) + 1), dict(scale=0.0), dict(scale=float("nan"))):
        assert call(**kw) == EINVAL, kw
    assert call(T=0) == 0 and call(B=0) == 0
    # few requests with long caches share a request's keys between workgroups, which takes a workspace
    need = agq.attn_kv_workspace_bytes(3, 4, 2, 128, 3, 1, 65536)
    assert need > 0 and need % (3 * 4 * (128 * 4 + 8)) == 0
    assert call(max_kv=65536) == EINVAL and call(max_kv=65536, ws=P + 8, wsb=need) == EINVAL
    assert call(max_kv=65536, ws=P, wsb=need - 1) == ESIZE


def test_workspace_sizes(agq):
    g = agq.attn_packed_workspace_bytes
    assert g(8192, 32, 8192, 8, 128, 1) == 0 and g(100, 32, 100, 8, 128, 1) == 0 and g(0, 32, 0, 8, 64, 0) == 0
    assert g(-1, 32, 9000, 8, 128, 1) == 0 and g(5, 3, 9000, 2, 128, 1) == 0 and g(5, 4, 9000, 2, 80, 1) == 0
    f = agq.attn_kv_workspace_bytes
    assert f(64, 32, 8, 128, 64, 1, 256) == 0                     # short: nothing is shared
    assert f(4096, 32, 8, 128, 4096, 1, 131072) == 0              # many requests: nothing to gain
    assert f(1, 32, 8, 128, 1, 1, 131072) > 0
    assert f(0, 32, 8, 128, 0, 1, 131072) == 0 and f(0, 32, 8, 128, 0, 0, 0) == 0
    for bad in ((-1, 32, 8, 128, 1, 1, 9), (1, 32, 5, 128, 1, 1, 9), (1, 32, 8, 96, 1, 1, 9), (1, 32, 8, 128, 70000, 1, 9), (1, 32, 8, 128, 1, -1, 9),
                (1, 32, 8, 128, 1, 1, -9)):
        assert f(*bad) == 0


def tensors():
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    c = lambda *s: torch.zeros(*s, dtype=torch.int8)
    return h, i, c


def test_binding_refuses_other_tensors(agq):
    h, i, c = tensors()
    kv = (c(6, 2, 16, 64), c(6, 2, 64, 16), c(6, 2), c(6, 2))
    cos = torch.zeros(8, 32)
    bad = [lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(4), *kv),                                   # slots of another batch
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3).long(), *kv),
           lambda: agq.kv_append(h(3, 2, 64).float(), h(3, 2, 64), i(3), *kv),
           lambda: agq.kv_append(h(3, 1, 64), h(3, 1, 64), i(3), *kv),
           lambda: agq.kv_append(h(3, 2, 64), h(2, 2, 64), i(3), *kv),
           lambda: agq.kv_append(h(3, 2, 128)[..., ::2], h(3, 2, 64), i(3), *kv),                        # strided inside a head
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv, q=h(3, 4, 64)),                    # rotation without tables
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv, pos=i(3), rope_cos=cos, rope_sin=cos[:, :16]),
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv, pos=i(3), rope_cos=cos, rope_sin=cos, q=h(2, 4, 64)),
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv, pos=i(3), rope_cos=cos, rope_sin=cos, k_out=h(3, 4, 64)),
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), kv[0], kv[0], kv[2], kv[3]),            # values that are not transposed
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), kv[0], kv[1], kv[2][:5], kv[3]),
           lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), kv[0], kv[1], kv[2].int(), kv[3]),
           lambda: agq.attn_kv(h(3, 4, 128), i(4), i(3), i(3, 2), *kv, 1, 32),
           lambda: agq.attn_kv(h(3, 4, 64), i(3), i(3), i(3, 2), *kv, 1, 32),
           lambda: agq.attn_kv(h(3, 4, 64), i(4), i(2), i(3, 2), *kv, 1, 32),
           lambda: agq.attn_kv(h(3, 4, 64), i(4), i(3), i(3, 4)[:, ::2], *kv, 1, 32),
           lambda: agq.attn_kv(h(3, 4, 64), i(4), i(3), i(3, 2), *kv, 1, 32, o=h(3, 2, 64)),
           lambda: agq.attn_packed(h(3, 4, 64), h(3, 2, 128), h(3, 2, 128), i(2), i(2)),
           lambda: agq.attn_packed(h(3, 4, 64), h(3, 2, 64), h(4, 2, 64), i(2), i(2)),
           lambda: agq.attn_packed(h(3, 4, 64), h(3, 2, 64), h(3, 2, 64), i(2), i(3)),
           lambda: agq.attn_packed(h(3, 4, 64), h(3, 2, 64), h(3, 2, 64), i(2), i(2), o=h(2, 4, 64)),
           lambda: agq.kv_map(i(3), i(2), i(3, 2), 16, i(6), i(2), 3),
           lambda: agq.kv_map(i(3), i(3), i(3, 2), 16, i(6), i(1), 3),
           lambda: agq.kv_map(i(3), i(3), i(3, 2).long(), 16, i(6), i(2), 3)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError("call %d was taken" % n)
    step = agq.KvStep(i(3), i(4), i(3), i(3), i(2), i(1))
    with pytest.raises(ValueError):
        agq.kv_map(i(3), i(3), i(3, 2), 16, i(6), i(2), 4, out=step)              # of another number of tokens


def test_binding_refuses_tensors_that_are_not_on_the_gpu(agq):
    """calls that are right but for their device"""
    h, i, c = tensors()
    kv = (c(6, 2, 16, 64), c(6, 2, 64, 16), c(6, 2), c(6, 2))
    cos = torch.zeros(8, 32)
    for call in (lambda: agq.kv_map(i(3), i(3), i(3, 2), 16, i(6), i(2), 3),
                 lambda: agq.kv_map(i(3), i(3), i(3, 2), 16, i(6), i(2), 3, out=agq.KvStep(i(3), i(4), i(3), i(3), i(2), i(1))),
                 lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv),
                 lambda: agq.kv_append(h(3, 2, 64), h(3, 2, 64), i(3), *kv, q=h(3, 4, 64), pos=i(3), rope_cos=cos, rope_sin=cos),
                 lambda: agq.attn_packed(h(3, 4, 64), h(3, 2, 64), h(3, 2, 64), i(2), i(2)),
                 lambda: agq.attn_kv(h(3, 4, 64), i(4), i(3), i(3, 2), *kv, 1, 32),
                 lambda: agq.attn_kv(h(3, 4, 64).to("meta"), i(4), i(3), i(3, 2), *kv, 1, 32)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


def test_oracle_attention_against_torch():
    """the yardstick of the GPU tests against torch's own float64 operators"""
    from oracle import agq_serve_oracle as so
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(n, 64, generator=g, dtype=torch.float64) for n in (7, 12, 12))
    sc = q @ k.t() / 8.0
    late = torch.arange(12)[None, :] > torch.arange(7)[:, None] + 5
    want = torch.softmax(sc.masked_fill(late, float("-inf")), -1) @ v
    got, bound = so.attention(q.numpy(), k.numpy(), v.numpy(), 5)
    assert abs(got - want.numpy()).max() < 1e-13 and (bound > 0).all() and bound.max() < 2e-2
    assert so.exponent(127.0) == 0 and so.exponent(127.5) == 1 and so.exponent(0) == -30 and so.exponent(float("inf")) == 10
    assert so.exponent(2.0 ** -24) == -30 and so.exponent(65504.0) == 10


@pytest.mark.parametrize("scale", [2.0 ** -61, 1e-38, 2.0 ** 24 * (1 + 2.0 ** -23), 1e30, 3e38])
def test_scales_out_of_range_are_refused(agq, scale):
    """scales with which scores would leave fp32's normal numbers"""
    assert agq.lib().agq_attn_packed(P, 512, 5, 4, P, 256, P, 256, 7, 2, 128, P, P, 2, 1, scale, P, 512, None, 0, None) == EINVAL
    assert agq.lib().agq_attn_kv(cache_of(), P, 512, 3, 4, P, P, 3, P, 4, 1, 64, scale, P, 512, None, 0, None) == EINVAL


def test_packed_refuses_more_workgroups_than_a_launch_has(agq):
    """a launch has less than 2^32 threads in a dimension: 2^24 workgroups of 256 are too many"""
    for Tq, B, H in ((1 << 20, 1 << 20, 32), (1 << 26, 1, 32), (1 << 19, 1 << 19, 32), (1 << 30, 1, 8), ((1 << 19) - 256, 1 << 19, 33)):
        assert agq.lib().agq_attn_packed(P, H * 64, Tq, H, P, 64, P, 64, 0, 1, 64, P, P, B, 1, 0.1, P, H * 64, None, 0, None) == EINVAL, (Tq, B, H)


def test_binding_refuses_half_a_rotation(agq):
    """rope_cos, rope_sin and pos without one of the others"""
    h, i, c = tensors()
    args, cos = (h(3, 2, 64), h(3, 2, 64), i(3), c(6, 2, 16, 64), c(6, 2, 64, 16), c(6, 2), c(6, 2)), torch.zeros(8, 32)
    for kw in (dict(rope_cos=cos), dict(rope_sin=cos), dict(pos=i(3)), dict(rope_cos=cos, rope_sin=cos), dict(rope_cos=cos, pos=i(3)),
               dict(rope_sin=cos, pos=i(3)), dict(rope_sin=cos, q=h(3, 4, 64))):
        with pytest.raises(ValueError, match="go with|go together"):
            agq.kv_append(*args, **kw)


def test_append_of_no_tokens_is_a_no_op(agq):
    """whatever is asked for: tensors of no tokens have no addresses"""
    call = lambda **kw: agq.lib().agq_kv_append(*dict(dict(cache=cache_of(), k=None, ldk=256, v=None, ldv=256, T=0, slot=None, q=None, ldq=512, Hq=4, pos=None,
                                                          cos=P, sin=P, rows=64, q_out=None, ldqo=512, k_out=None, ldko=256, stream=None), **kw).values())
    assert call() == 0 and call(Hq=0) == 0 and call(q=P, k_out=P) == 0
    assert call(Hq=-1) == EINVAL and call(cache=None) == EINVAL and call(T=5) == EINVAL
