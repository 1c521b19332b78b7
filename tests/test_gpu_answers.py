"""Log probabilities, entropies and likeliest tokens on the GPU against their definition in float64, within the bound that
float32 arithmetic allows (oracle/agq_serve_oracle.py); the tokens themselves exactly."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import agq_serve_oracle as so  # noqa: E402
from test_gpu_parity import dev, host  # noqa: E402

TYPES = {"fp16": np.float16, "fp32": np.float32}
SENTINEL = 77.0


@pytest.fixture(scope="module")
def agq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2312_05693_amd import binding
    binding.lib()
    return binding


def draw(r, T, V, kind, spread=2.5):
    x = r.standard_normal((T, V)) * spread
    for t in range(T):
        x[t, r.integers(0, V, 4)] += r.uniform(3, 12, 4)
    return x.astype(TYPES[kind])


def compare(got, want, n_top, label=""):
    for name, bound in (("logprob", "logprob_bound"), ("entropy", "entropy_bound"), ("top_logprob", "top_bound")):
        g = getattr(got, name)
        if g is None:
            assert name == "top_logprob" and n_top == 0
            continue
        g, w = host(g).astype(np.float64), want[name]
        assert np.array_equal(np.isnan(g), np.isnan(w)), (label, name)
        # float32 ends at 2^128 (1 - 2^-24); what is 2^128 (1 - 2^-25) or more rounds to infinity
        w = np.where(np.abs(w) >= 2.0 ** 128 - 2.0 ** 103, np.copysign(np.inf, w), w)
        inf = np.isinf(w)
        assert np.array_equal(g[inf], w[inf]), (label, name)
        fine = np.isfinite(w)
        off = np.abs(g[fine] - w[fine]) - want[bound][fine]
        assert (off <= 0).all(), (label, name, off.max(), want[bound][fine][off.argmax()])
    if n_top:
        assert np.array_equal(host(got.top_idx), want["top_idx"]), label


def check(agq, x, tokens, n_top, scale=1.0, logits=None):
    """logits: the tensor to pass in, if it is not simply x"""
    got = agq.logprobs(dev(x) if logits is None else logits, dev(np.asarray(tokens, np.int32)), n_top=n_top, scale=scale)
    compare(got, so.logprobs(x, tokens, n_top, np.float32(scale)), n_top)
    return got


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 2047, 2049, 4097, 8191, 8192, 8200, 32000])
@pytest.mark.parametrize("T,n_top", [(1, 5), (3, 0), (9, 64), (2, 1)])
def test_sizes(agq, kind, V, T, n_top):
    r = np.random.default_rng([V, T, n_top])
    check(agq, draw(r, T, V, kind), r.integers(0, V, T), min(n_top, V))


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("T,V,n_top", [(1, 131072, 20), (5, 128000, 64), (40, 50001, 8), (300, 4001, 10), (1500, 1000, 3), (700, 32000, 20),
                                       (2, 1 << 20, 33), (200, 70001, 20), (256, 128000, 0), (130, 300001, 7), (600, 300001, 2), (257, 32769, 64)])
def test_large(agq, kind, T, V, n_top):
    r = np.random.default_rng([V, T])
    check(agq, draw(r, T, V, kind), r.integers(0, V, T), n_top)


def test_largest_vocabulary(agq):
    r = np.random.default_rng(1)
    V = 1 << 24
    x = (r.standard_normal((1, V), dtype=np.float32) * 2).astype(np.float16)
    check(agq, x, [V - 1], 20)


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("V,pad,shift", [(1000, 1, 1), (4097, 3, 0), (129, 6, 5), (32001, 0, 0), (50001, 7, 3)])
def test_rows_at_any_distance_and_place(agq, kind, V, pad, shift):
    """rows that begin at odd elements; what lies between and around them is infinite and NaN"""
    r = np.random.default_rng([V, pad])
    T = 6
    x = draw(r, T, V, kind)
    wide = np.full((T, shift + V + pad), np.inf, dtype=x.dtype)
    wide[::2] = np.nan
    wide[:, shift:shift + V] = x
    d = dev(wide)
    check(agq, x, r.integers(0, V, T), min(V, 9), logits=d[:, shift:shift + V])


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("V", [100, 5000, 40000])
@pytest.mark.parametrize("n_top", [1, 20, 64])
def test_equal_logits_go_by_their_index(agq, kind, V, n_top):
    r = np.random.default_rng([V, n_top])
    rows = [np.zeros(V), r.integers(0, 3, V), np.where(r.random(V) < 0.5, 0.0, -0.0), np.repeat(r.standard_normal(V // 50 + 1), 50)[:V],
            np.full(V, -3.0), np.arange(V) // 300 * 0.125, -(np.arange(V) // 300) * 0.125, np.sort(r.standard_normal(V)), -np.sort(r.standard_normal(V)),
            np.where(np.arange(V) == V - 1, 5.0, 1.0)]
    x = np.stack(rows).astype(TYPES[kind])
    check(agq, x, r.integers(0, V, len(x)), n_top)


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("V", [70, 3001, 40000, 131072])
def test_tokens_that_are_ruled_out(agq, kind, V):
    """-infinity nearly everywhere; rows that nothing, +infinity or a NaN leaves without a distribution, beside good ones"""
    r = np.random.default_rng(V)
    x = draw(r, 12, V, kind)
    x[1, 3:] = -np.inf
    x[2] = -np.inf
    x[3, :V - 1] = -np.inf
    x[4] = np.where(r.random(V) < 0.99, -np.inf, x[4])
    x[4, V // 2] = 1
    x[5, V // 3] = np.inf
    x[6, V - 1] = np.nan
    x[7, 0] = -np.nan
    x[8] = -np.inf
    x[8, V // 2] = -60000.0
    x[9, ::2] = -np.inf
    x[10] = np.where(np.arange(V) < V // 2, -np.inf, 0.25)
    tokens = [0, 5, 1, V - 1, V // 2, V // 3, 0, 9, V // 2, 0, V // 2 - 1, 7]
    for n_top in (0, 5, 64):
        got = check(agq, x, tokens, n_top)
        assert host(got.logprob)[9] == -np.inf and host(got.logprob)[8] == 0 and host(got.entropy)[8] == 0


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("scale", [2.0 ** -24, 1e-3, 0.7, 37.7, 2.0 ** 24])
def test_scales_and_large_logits(agq, kind, scale):
    r = np.random.default_rng(6)
    V = 3000
    x = draw(r, 6, V, kind)
    x[1] = (r.standard_normal(V) * 60000).clip(-65504, 65504)
    x[2, 5] = 65504
    x[3] = -65504
    x[4] = x[4] * 1e-4
    check(agq, x, r.integers(0, V, 6), 12, scale)


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("V", [300, 50001])
def test_masks_of_the_lowest_value(agq, kind, scale, V):
    """differences from it, times the scale in bits, are beyond float32"""
    r = np.random.default_rng([9, V])
    low = np.finfo(TYPES[kind]).min
    x = draw(r, 6, V, kind)
    x[0, r.random(V) < 0.5] = low
    x[1, 3:] = low                                       # fewer tokens left than are asked for
    x[2] = low
    x[3] = low
    x[3, V // 2] = -np.inf
    x[4, 7:] = np.where(r.random(V - 7) < 0.5, low, -np.inf)
    x[5] = low
    x[5, 7] = -low
    check(agq, x, [int(np.argmin(x[0])), 2, 0, V // 2, 8, 7], 12, scale)


def test_sure_answers(agq):
    """one logit far above the others: entropy and the loss are small, not lost in the sum's rounding"""
    x = np.zeros((4, 2000), np.float32)
    for t, up in enumerate((12.0, 25.0, 80.0, 1000.0)):
        x[t, 17] = up
    check(agq, x, [17, 17, 17, 17], 3)


def test_tokens_out_of_range_and_results_not_asked_for(agq):
    r = np.random.default_rng(8)
    x = draw(r, 5, 777, "fp16")
    got = check(agq, x, [0, -1, 777, 776, 2 ** 31 - 1], 4)
    assert np.isnan(host(got.logprob)).tolist() == [False, True, True, False, True]
    only = agq.logprobs(dev(x), n_top=4, want_entropy=False)
    assert only.logprob is None and only.entropy is None and torch.equal(only.top_idx, got.top_idx) and torch.equal(only.top_logprob, got.top_logprob)
    one = agq.logprobs(dev(x), dev(np.zeros(5, np.int32)), want_entropy=False)
    assert one.top_idx is None and one.entropy is None and host(one.logprob)[0] == host(got.logprob)[0]
    ent = agq.logprobs(dev(x))
    assert ent.logprob is None and torch.equal(ent.entropy, got.entropy)
    none = agq.logprobs(dev(x), want_entropy=False)
    assert none == (None, None, None, None)
    assert agq.logprobs(dev(x[:0]), dev(np.zeros(0, np.int32)), n_top=2).top_idx.shape == (0, 2)


def test_results_lie_where_they_should(agq):
    """nothing is written in front of or behind the results"""
    r = np.random.default_rng(9)
    T, V, n = 7, 1234, 6
    x = draw(r, T, V, "fp16")
    whole = torch.full((3, T * n + 20), SENTINEL, device="cuda")
    idx = torch.full((T * n + 20,), -9, dtype=torch.int32, device="cuda")
    out = agq.Logprobs(whole[0, 10:10 + T], whole[1, 10:10 + T], idx[10:10 + T * n].view(T, n), whole[2, 10:10 + T * n].view(T, n))
    tokens = r.integers(0, V, T)
    got = agq.logprobs(dev(x), dev(tokens.astype(np.int32)), n_top=n, out=out)
    compare(got, so.logprobs(x, tokens, n), n)
    for row, used in ((whole[0], T), (whole[1], T), (whole[2], T * n)):
        row = host(row)
        assert (row[:10] == SENTINEL).all() and (row[10 + used:] == SENTINEL).all()
    assert (host(idx)[:10] == -9).all() and (host(idx)[10 + T * n:] == -9).all()


def test_rows_a_gigabyte_apart(agq):
    """offsets that pass 32 bits"""
    r = np.random.default_rng(10)
    V, ld = 5000, 1 << 30
    x = draw(r, 4, V, "fp16")
    store = torch.empty(3 * ld + V, dtype=torch.float16, device="cuda")
    view = store.as_strided((4, V), (ld, 1))
    view.copy_(dev(x))
    check(agq, x, r.integers(0, V, 4), 20, logits=view)


@pytest.mark.parametrize("T,V,n_top", [(2, 128000, 20), (600, 2000, 5)])
def test_workspaces_refused(agq, T, V, n_top):
    need = agq.logprobs_workspace_bytes(T, V, 0, n_top)
    if need == 0:
        return
    x = torch.zeros(T, V, dtype=torch.float16, device="cuda")
    with pytest.raises(agq.AgqError) as e:
        agq.logprobs(x, n_top=n_top, workspace=torch.empty(need - 1, dtype=torch.int8, device="cuda"))
    assert e.value.status == agq.AGQ_ESIZE
    with pytest.raises(ValueError):
        agq.logprobs(x, n_top=n_top, workspace=torch.empty(need, dtype=torch.int8))


@pytest.mark.parametrize("T,V,n_top", [(3, 50001, 20), (700, 3000, 4)])
def test_captured_and_replayed(agq, T, V, n_top):
    """replays with other logits between them, the results of each against an eager call"""
    r = np.random.default_rng(11)
    x, tok = dev(draw(r, T, V, "fp16")), dev(r.integers(0, V, T).astype(np.int32))
    ws = torch.empty(max(16, agq.logprobs_workspace_bytes(T, V, 0, n_top)), dtype=torch.int8, device="cuda")
    eager = agq.logprobs(x, tok, n_top=n_top)
    out = agq.Logprobs(*[torch.empty_like(t) for t in eager])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        agq.logprobs(x, tok, n_top=n_top, out=out, workspace=ws)
    for n in range(4):
        data = draw(r, T, V, "fp16")
        x.copy_(dev(data))
        ws.random_(-128, 127)
        want = agq.logprobs(x, tok, n_top=n_top)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), n
        if n == 0:
            compare(out, so.logprobs(data, host(tok), n_top), n_top)


def test_two_streams_at_once(agq):
    r = np.random.default_rng(12)
    jobs = [(dev(draw(r, T, V, k)), dev(r.integers(0, V, T).astype(np.int32)), n) for T, V, k, n in ((4, 128000, "fp16", 20), (300, 9000, "fp32", 7))]
    want = [agq.logprobs(x, t, n_top=n) for x, t, n in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i, (s, (x, t, n)) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[i].append(agq.logprobs(x, t, n_top=n))
    torch.cuda.synchronize()
    for i in range(2):
        for res in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(res, want[i]))


def test_logits_of_the_quantized_layer(agq):
    """from a hidden state through the 4-bit output layer to scores, as a program scores a text"""
    from paper_2312_05693_amd import synth
    M, K, N = 33, 256, 4096
    x = synth.make_activation(M, K, 2, 3)
    wq, sw = synth.make_weight_q4(N, K, 3)
    e = int(agq.calibrate_act_exp(dev(x), 8).item())
    y = agq.gemm_w4a8(dev(x), e, agq.pack_w4(dev(wq)), dev(sw), N, K)
    tokens = np.arange(M) * 100
    got = agq.logprobs(y, dev(tokens.astype(np.int32)), n_top=5)
    compare(got, so.logprobs(host(y), tokens, 5), 5)


def even_rows(V, kind):
    """rows whose logits are nearly equal: a sum of them, one after the other in float32, is off by the same way at every step"""
    rows, n = [], min(V, 2048)
    for up in (0.3, 1.0, 2.5):                       # a few larger ones in front of every quarter
        x = np.zeros(V)
        for q in range(4):
            x[q * V // 4:q * V // 4 + n] = up
        rows.append(x)
    rows += [np.linspace(0.0, 0.5, V), np.linspace(2.0, 0.0, V), np.linspace(-3.0, 3.0, V), np.full(V, 1.5)]
    return np.stack(rows).astype(TYPES[kind])


def check_even(agq, kind, T, V, n_top, scale):
    """against float64 within the bounds of include/agq.h, which do not know V"""
    x = even_rows(V, kind)
    at = np.arange(T) % len(x)
    tokens = np.array([0, V - 1, V // 2, V // 3, 0, V - 1, 1], dtype=np.int32)[:len(x)]
    logits = dev(x)[torch.from_numpy(at).cuda()]
    got = agq.logprobs(logits, dev(tokens[at]), n_top=n_top, scale=scale)
    lp, ent, d = host(got.logprob).astype(np.float64), host(got.entropy).astype(np.float64), 2.0 ** -24
    for i in range(min(T, len(x))):
        y = x[i].astype(np.float64)
        z = (y - y.max()) * float(np.float32(scale))
        lse = np.log(np.exp(z).sum())
        p = np.exp(z - lse)
        want, H = z[tokens[i]] - lse, -(p * (z - lse)).sum()
        D, Q = (p * -z).sum(), (p * z * z).sum()
        off = abs(lp[i] - want), abs(ent[i] - H)
        assert off[0] <= d * (abs(want) + 8 * D + 32) and off[1] <= d * (H + 128 + 128 * D + 16 * Q), (i, off, D, Q)
        assert (lp[at == i] == lp[i]).all() and (ent[at == i] == ent[i]).all()
        if n_top:
            best = np.argsort(-y, kind="stable")[:n_top]
            assert np.array_equal(host(got.top_idx)[i], best)
            assert (np.abs(host(got.top_logprob)[i] - (z[best] - lse)) <= d * (np.abs(z[best] - lse) + 8 * D + 32)).all()


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("scale", [1.0, 0.37])
@pytest.mark.parametrize("T,V,n_top", [(300, 32000, 0), (300, 131072, 0), (600, 131072, 3), (140, 131072, 0), (1, 131072, 2), (7, 1 << 20, 0),
                                       (300, 1 << 20, 0), (520, 1 << 20, 2)])
def test_rows_of_nearly_equal_logits(agq, kind, scale, T, V, n_top):
    check_even(agq, kind, T, V, n_top, scale)


def test_long_rows_of_nearly_equal_logits(agq):
    check_even(agq, "fp16", 513, 1 << 24, 0, 1.0)
    check_even(agq, "fp16", 2, 1 << 24, 1, 1.0)


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("T,V,n_top", [(3, 300001, 7), (40, 70001, 8), (3, 70001, 0), (600, 600001, 2)])
def test_workspaces_that_are_needed(agq, kind, T, V, n_top):
    """rows in pieces: a workspace that is too small, elsewhere or odd is refused, one of the least size is enough, and nothing
    behind it is written"""
    need = agq.logprobs_workspace_bytes(T, V, {"fp16": 0, "fp32": 1}[kind], n_top)
    assert need > 0
    row = np.random.default_rng([T, V]).standard_normal((2, V)).astype(TYPES[kind])
    logits = dev(row)[torch.arange(T, device="cuda") % 2]
    store = torch.full((need + 64,), 85, dtype=torch.int8, device="cuda")
    for bad, status in ((store[:need - 1], agq.AGQ_ESIZE), (store[8:8 + need], agq.AGQ_EINVAL)):
        with pytest.raises(agq.AgqError) as e:
            agq.logprobs(logits, n_top=n_top, workspace=bad)
        assert e.value.status == status
    with pytest.raises(ValueError):
        agq.logprobs(logits, n_top=n_top, workspace=torch.empty(need, dtype=torch.int8))
    assert (store == 85).all()
    got = agq.logprobs(logits, dev(np.zeros(T, np.int32)), n_top=n_top, workspace=store[:need])
    assert (store[need:] == 85).all() and bool((store[:need] != 85).any())
    want = so.logprobs(row, [0, 0], n_top)
    at = np.arange(T) % 2
    compare(got, {k: v[at] for k, v in want.items()}, n_top)
