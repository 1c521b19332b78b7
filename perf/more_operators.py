"""Operators that a program which serves a model needs beside the cache and its attentions, as cases that can be timed and
compared: what the model's answers are worth (log probabilities and the likeliest tokens), requests that become several or
lose tokens (forks and compactions of the paged cache), and models whose queries and keys are normalised per head.

A case is a dict of plain values; its "kind" says which operator it runs:

  score    the log probability of a given token in every row of logits, the row's entropy, and its n_top likeliest tokens
           with their log probabilities (binding.logprobs)
  norm     queries and keys normalised per head and turned by their positions, in fp16 (binding.qk_norm_rope)
  append   the same on the way into the paged 8-bit cache (binding.kv_append_norm)
  fork     requests that go on as copies of others: full pages are shared, partly filled ones copied in every layer, pages
           that nobody holds any more go back (binding.kv_fork, binding.kv_copy_pages)
  compact  requests that lose tokens in their midst or at their end: what is left moves together, in every layer
           (binding.kv_compact, binding.kv_move)

Sizes are those of the LLaMA-7B and -13B shapes and the 768-wide layer that the tests and the benchmark of this repository
use, with all heads of their own or in groups of two to eight, and vocabularies of some thousands to 131072 tokens."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
ROPE_BASE = 10000.0
E_ZERO = -30            # exponent of a page that holds zeros only: the smallest that a page can have
MAX_POSITION = 8192     # rows of the rotary tables
EPS = 1e-6
CACHE_BYTES = 400e6     # of all layers of a fork's or a compaction's cache


def listed():
    return [
        # one user's token: five alternatives of a small vocabulary, the smallest call
        dict(name="score_1", kind="score", T=1, V=32000, type="fp16", n_top=5, masked=0),
        # a generation step of a busy server, a large vocabulary
        dict(name="score_step_64", kind="score", T=64, V=128000, type="fp16", n_top=20, masked=0),
        # answers held to a grammar: most of the vocabulary is ruled out in some rows; an odd vocabulary, float32 logits
        dict(name="score_grammar_200", kind="score", T=200, V=50001, type="fp32", n_top=8, masked=60),
        # a text is scored: no alternatives, every row
        dict(name="score_text_4096", kind="score", T=4096, V=32000, type="fp16", n_top=0, masked=0),
        # one user's token in the 7B shape
        dict(name="norm_7b_1", kind="norm", T=1, Hq=32, Hkv=32, D=128, own_gains=0),
        # prompts of the 13B shape that are only scored (no cache)
        dict(name="norm_13b_6000", kind="norm", T=6000, Hq=40, Hkv=40, D=128, own_gains=0),
        # a generation step of a busy server, grouped heads
        dict(name="append_norm_step_256", kind="append", T=256, B=256, Hq=32, Hkv=8, D=128, page=64, new="step"),
        # prompts of many lengths, heads of 64
        dict(name="append_norm_prompts", kind="append", T=7001, B=11, Hq=32, Hkv=8, D=64, page=64, new="prompts"),
        # a beam search of a few prompts moves on by a token
        dict(name="fork_beams_8", kind="fork", B=8, width=4, longest=500, Hkv=8, D=128, page=16, layers=32, new="beams"),
        # prompts of a busy server are answered several times each
        dict(name="fork_samples_256", kind="fork", B=256, width=8, longest=1500, Hkv=8, D=64, page=64, layers=8, new="samples"),
        # drafts were checked: requests lose some of their last tokens
        dict(name="compact_drafts_64", kind="compact", B=64, longest=1000, Hkv=8, D=128, page=64, layers=4, new="drafts"),
        # long contexts lose half of their tokens, some prompts are shared
        dict(name="compact_prune_8", kind="compact", B=8, longest=16384, Hkv=8, D=128, page=64, layers=2, new="prune"),
    ]


def _spread(rng, lo, hi):
    """a whole number in [lo, hi], spread over its logarithm"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 12, 32, 40])
    group = rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * Hkv <= 40])
    return dict(Hq=group * Hkv, Hkv=Hkv, D=D)


def draw(rng):
    kind = rng.choice(["score", "norm", "append", "fork", "compact"])
    if kind == "score":
        V = _spread(rng, 1000, 131072)
        type_ = rng.choice(["fp16", "fp16", "fp32"])
        T = _spread(rng, 1, min(4096, (130_000_000 if type_ == "fp16" else 65_000_000) // V))
        return dict(kind=kind, T=T, V=V, type=type_, n_top=rng.choice([0, 1, 5, 10, 20, 33, 64]),
                    masked=rng.choice([0, 0, 30]))
    if kind == "norm":
        return dict(kind=kind, T=_spread(rng, 1, 6000), own_gains=rng.choice([0, 0, 1]), **_heads(rng))
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        new = rng.choice(["step", "prompts"])
        B = _spread(rng, 1, 256)
        T = B if new == "step" else max(B, _spread(rng, 8, 4000))
        return dict(kind=kind, T=T, B=B, page=page, new=new, **_heads(rng))
    Hkv, D, layers = rng.choice([1, 2, 5, 8, 12]), rng.choice([64, 128]), rng.choice([1, 2, 5, 12, 32])
    tokens = int(CACHE_BYTES / (2 * Hkv * D * layers))               # that the cache has room for
    if kind == "fork":
        width = rng.choice([2, 4, 5, 8])
        B = width * _spread(rng, 1, max(1, min(256, tokens // (4 * page)) // width))
        return dict(kind=kind, B=B, width=width, longest=_spread(rng, 16, max(17, min(4096, tokens // (2 * B)))), Hkv=Hkv, D=D, page=page,
                    layers=layers, new=rng.choice(["beams", "samples"]))
    B = _spread(rng, 1, max(2, min(64, tokens // (8 * page))))
    return dict(kind=kind, B=B, longest=_spread(rng, 32, max(33, min(16384, tokens // (2 * B)))), Hkv=Hkv, D=D, page=page, layers=layers,
                new=rng.choice(["drafts", "prune"]))


# ------------------------------------------------------------------ sizes of a case, from the case alone

def _numbers(case, tag):
    return np.random.default_rng([int(sum(ord(c) * (i + 7) for i, c in enumerate(repr(sorted((k, v) for k, v in case.items()
                                                                                           if k != "name"))))), tag])


def _pages(n, page):
    return (np.asarray(n, dtype=np.int64) + page - 1) // page


def _append_sizes(case):
    r, B, T = _numbers(case, 2), case["B"], case["T"]
    if case["new"] == "step":
        return r.integers(0, 2000, B), np.ones(B, dtype=np.int64)
    cuts = np.sort(r.integers(0, T - B + 1, B - 1))
    new = np.diff(np.concatenate([[0], cuts, [T - B]])) + 1
    past = np.where(r.uniform(0, 1, B) < 0.7, 0, r.integers(1, 500, B))
    return np.minimum(past, np.maximum(0, MAX_POSITION - new)), new


def _fork_sizes(case):
    """Lengths, the common prompts' lengths, and parents.  Requests stand in families of `width`.  beams: all of them live
    and share the full pages of their prompt; each goes on as one of its family, one family in eight has ended.  samples:
    the first one of a family lives, and all of them go on as it."""
    r, B, W = _numbers(case, 4), case["B"], case["width"]
    fam = np.arange(B) // W
    n_fam = int(fam[-1]) + 1
    prompt = np.exp(r.uniform(math.log(8), math.log(case["longest"]), n_fam)).astype(np.int64)
    prompt[0] = case["longest"]
    if case["new"] == "samples":
        length = np.where(np.arange(B) % W == 0, prompt[fam], 0)
        return length, prompt[fam], fam * W
    length = prompt[fam] + r.integers(1, 2 * case["page"], n_fam)[fam]                 # as many new tokens for all of a family
    parent = fam * W + r.integers(0, W, B)
    ended = (np.arange(n_fam) % 8 == 7)[fam]
    return length, prompt[fam], np.where(ended, -1, np.minimum(parent, B - 1))


def _compact_sizes(case):
    """Lengths, the number of first tokens that stay, how many of the others are kept, and the first tokens that a request
    shares with the one before it."""
    r, B = _numbers(case, 5), case["B"]
    length = np.exp(r.uniform(math.log(16), math.log(case["longest"] + 0.5), B)).astype(np.int64)
    length[0] = case["longest"]
    if case["new"] == "drafts":
        drafts = np.minimum(8, length - 1)
        stay = length - drafts
        tree = r.uniform(0, 1, B) < 0.3                                                # some of the drafted tokens, not the first ones
        stay = np.where(tree, stay, stay + r.integers(0, 9, B).clip(0, drafts))
        kept = np.where(tree, np.minimum(r.integers(1, 5, B), drafts), 0)
        return length, stay, kept, np.zeros(B, dtype=np.int64)
    stay = np.minimum(r.integers(1, 2 * case["page"], B), length)
    kept = (length - stay) // 2
    common = np.where(np.arange(B) % 4 == 1, np.minimum(length, np.roll(length, 1)) // 2, 0)
    return length, stay, kept, common // case["page"] * case["page"]


def work(case):
    kind = case["kind"]
    if kind == "score":
        T, V, n = case["T"], case["V"], case["n_top"]
        # logits and tokens in; log probability, entropy and alternatives out.  A difference, a product, an exponential, two sums
        return {"bytes": T * (V * (2 if case["type"] == "fp16" else 4) + 4 + 8 + 8 * n), "flops": 6 * T * V}
    if kind in ("norm", "append"):
        T, Hq, Hkv, D = (case[n] for n in ("T", "Hq", "Hkv", "D"))
        if kind == "norm":
            # q and k in and out; a position, its angles, the gains
            return {"bytes": T * (4 * D * (Hq + Hkv) + 4 + 4 * D) + 4 * D, "flops": T * D * 7 * (Hq + Hkv)}
        return {"bytes": T * (2 * D * (2 * Hq + 3 * Hkv) + 2 * D * Hkv + 8 + 4 * D) + 4 * D, "flops": T * D * (7 * Hq + 9 * Hkv)}
    page, row = case["page"], case["layers"] * 2 * case["Hkv"] * case["D"]             # bytes of a token in all layers
    if kind == "fork":
        length, _, parent = _fork_sizes(case)
        after = np.where(parent >= 0, length[parent], 0)
        copies = sum(int((parent == p).sum()) - 1 for p in np.unique(parent[parent >= 0]) if length[p] % page)
        # the tokens of partly filled pages, to be read and written; lengths, parents, page numbers, holders' counts
        some = sum(int(length[p] % page) * (int((parent == p).sum()) - 1) for p in np.unique(parent[parent >= 0]))
        return {"bytes": 2 * some * row + 4 * copies * case["layers"] * case["Hkv"] + 4 * (3 * case["B"] + int(2 * _pages(after, page).sum())),
                "flops": 2 * int(_pages(after, page).sum())}
    length, stay, kept, _ = _compact_sizes(case)
    moved = kept + np.where(kept > 0, stay % page, 0)
    # tokens of new pages, read and written, and where they are; lengths, page numbers
    return {"bytes": int(2 * moved.sum()) * row + 4 * int(kept.sum()) + 4 * (3 * case["B"] + int(2 * _pages(stay + kept, page).sum())),
            "flops": int(moved.sum()) * row}


# ------------------------------------------------------------------ what a program has in hand

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _int32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _sums(n):
    return np.concatenate([[0], np.cumsum(n)])


def _tables(D):
    angle = np.arange(MAX_POSITION, dtype=np.float64)[:, None] * ROPE_BASE ** (-2.0 * np.arange(D // 2) / D)[None, :]
    return (torch.from_numpy(np.cos(angle).astype(np.float32)).to(DEVICE), torch.from_numpy(np.sin(angle).astype(np.float32)).to(DEVICE))


def _random_cache(g, n_pages, Hkv, page, D):
    """Pages as earlier steps left them: codes of normal values, whose scales differ by a few powers of two."""
    def codes(*shape):
        return (_normal(g, *shape) * 40.0).round_().clamp_(-127, 127).to(torch.int8)

    def exps():
        return torch.randint(-7, -4, (n_pages, Hkv), generator=g, device=DEVICE, dtype=torch.int32).to(torch.int8)
    return codes(n_pages, Hkv, page, D), codes(n_pages, Hkv, D, page), exps(), exps()


def _gains(g, heads, D, own_gains):
    return (1.0 + 0.1 * _normal(g, *((heads, D) if own_gains else (D,)))).half()


def _prepare_score(case, g, st):
    T, V = case["T"], case["V"]
    x = _normal(g, T, V) * 2.5
    likely = torch.randint(0, V, (T, 12), generator=g, device=DEVICE)
    x.scatter_add_(1, likely, 6.0 + 4.0 * torch.rand(T, 12, generator=g, device=DEVICE))
    if case["masked"]:
        # rows with a grammar: all but a few tokens are ruled out, in some of them all but one or two
        few = torch.rand(T, 1, generator=g, device=DEVICE)
        share = torch.where(few < 0.1, 1.5 / V, torch.where(few < 0.01 * case["masked"], 0.01, 2.0))
        out = torch.rand(T, V, generator=g, device=DEVICE) >= share
        out.scatter_(1, likely[:, :1], False)
        x.masked_fill_(out, -math.inf)
    st["logits"] = x.half() if case["type"] == "fp16" else x
    st["tokens"] = torch.where(torch.rand(T, generator=g, device=DEVICE) < 0.7, likely[:, 0],
                               torch.randint(0, V, (T,), generator=g, device=DEVICE)).int()


def _prepare_heads(case, g, r, st):
    Hq, Hkv, D, T = (case[n] for n in ("Hq", "Hkv", "D", "T"))
    # one tensor holds q, k and v of a token side by side, as one projection writes them; a few channels are larger
    qkv = (_normal(g, T, Hq + 2 * Hkv, D) * (1.0 + 7.0 * (torch.rand(1, Hq + 2 * Hkv, D, generator=g, device=DEVICE) < 0.02))).half()
    cos, sin = _tables(D)
    per_head = case.get("own_gains", 0)
    st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], cos=cos, sin=sin, g_q=_gains(g, Hq, D, per_head),
              g_k=_gains(g, Hkv, D, per_head))
    if case["kind"] == "norm":
        st["pos"] = _int32((np.arange(T) + r.integers(0, MAX_POSITION)) % MAX_POSITION)
        return
    page = case["page"]
    past, new = _append_sizes(case)
    most = _pages(past + new, page)
    n_pages = int(most.sum()) + 8
    ids = r.permutation(n_pages)
    first = _sums(most)
    pos = np.concatenate([p + np.arange(n) for p, n in zip(past, new)])
    of = np.repeat(np.arange(case["B"]), new)
    kc, vc, ke, ve = _random_cache(g, n_pages, Hkv, page, D)
    st.update(pos=_int32(pos), slot=_int32(ids[first[of] + pos // page] * page + pos % page), k_cache=kc, v_cache=vc, k_exp=ke, v_exp=ve)


def _pool(case, g, r, st, length, common, needed):
    """Pages dealt out at random (the first common[b] tokens' pages of a request are those of the request before it),
    the counts of their further holders, the ring of the free ones, and the caches of all layers."""
    page, B, L = case["page"], case["B"], case["layers"]
    held, before = _pages(length, page), np.asarray(common) // page
    n_pages = int((held - before).sum()) + needed + 5
    ids = r.permutation(n_pages)
    table, shared, at = np.full((B, int(max(held.max(), 1)) + 1), -1, dtype=np.int32), np.zeros(n_pages, dtype=np.int32), 0
    for b in range(B):
        n = int(before[b])
        if n:
            table[b, :n] = table[b - 1, :n]
            shared[table[b, :n]] += 1
        table[b, n:held[b]] = ids[at:at + held[b] - n]
        at += int(held[b]) - n
    ring, head = np.full(n_pages, -1, dtype=np.int32), int(r.integers(0, n_pages))
    ring[(head + np.arange(n_pages - at)) % n_pages] = ids[at:]
    # the layers' caches lie in one tensor of each kind
    whole = [torch.cat(parts).view(L, n_pages, *parts[0].shape[1:])
             for parts in zip(*(_random_cache(g, n_pages, case["Hkv"], page, case["D"]) for _ in range(L)))]
    st.update(kv_len=_int32(length), table=_int32(table), shared=_int32(shared), ring=_int32(ring), free=_int32([head, n_pages - at]), page=page,
              whole=whole, caches=list(zip(*whole)))
    # what a program that swaps two of each from step to step has ready
    new = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEVICE)
    st["out"] = dict(kv_len=new(B), block_table=torch.full_like(st["table"], -1), shared=new(n_pages), copy_src=new(B), copy_dst=new(B),
                     free_state=new(2), status=new(1))


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed) + 1)
    r = np.random.default_rng([int(seed), 9])
    st = dict(case=case, kind=case["kind"])
    if case["kind"] == "score":
        _prepare_score(case, g, st)
        return st
    if case["kind"] in ("norm", "append"):
        _prepare_heads(case, g, r, st)
        return st
    B, page = case["B"], case["page"]
    if case["kind"] == "fork":
        length, prompt, parent = _fork_sizes(case)
        first = np.arange(B) % case["width"] == 0
        common = np.where(first | (case["new"] == "samples"), 0, prompt)
        _pool(case, g, r, st, length, common // page * page, B)
        st["parent"] = _int32(parent)
    else:
        length, stay, kept, common = _compact_sizes(case)
        keep = [np.sort(r.choice(int(n - s), int(k), replace=False)) + s for n, s, k in zip(length, stay, kept)]
        _pool(case, g, r, st, length, common, int((_pages(kept, page) + 2).sum()))
        st.update(stay=_int32(stay), cu_keep=_int32(_sums(kept)), keep=_int32(np.concatenate(keep) if sum(kept) else np.zeros(0)))
    if own:
        from paper_2312_05693_amd import binding as agq
        st["layers"] = agq.kv_layers(st["caches"])                                     # addresses of the layers' caches, made once
        o = st["out"]
        if case["kind"] == "fork":
            st["step"] = agq.KvFork(o["kv_len"], o["block_table"], o["shared"], o["copy_src"], o["copy_dst"], o["free_state"], o["status"])
        else:
            o["moves"] = torch.zeros(agq.kv_moves_ints(st["keep"].numel(), B, page), dtype=torch.int32, device=DEVICE)
            st["step"] = agq.KvCompact(o["kv_len"], o["block_table"], o["shared"], o["moves"], o["free_state"], o["status"])
    return st


# ------------------------------------------------------------------ the plain forms

def _plain_score(s):
    x, n = s["logits"].float(), s["case"]["n_top"]
    top = x.amax(1, keepdim=True)
    d = x - top
    p = torch.exp(d)
    total = p.sum(1, keepdim=True)
    logs = d - torch.log(total)
    p /= total
    entropy = -torch.where(p > 0, p * logs, torch.zeros_like(p)).sum(1)
    out = [logs.gather(1, s["tokens"].long()[:, None])[:, 0], entropy]
    if n:
        # larger values first, equal ones by their index: both in one whole number
        bits = (x + 0.0).view(torch.int32)
        bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
        key = (bits.long() << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device=DEVICE))
        index = x.shape[1] - 1 - (torch.topk(key, n, dim=1).values & 0xFFFFFFFF)
        out += [index.int(), logs.gather(1, index)]
    return out


def _round_once(x):
    """float64 -> fp16 with one rounding: to float32 by truncation with the last bit set where anything was cut off,
    which the second rounding then sees."""
    f = x.float()
    u = f.view(torch.int32)
    u = u - (f.double().abs() > x.abs()).int()
    return torch.where(f.double() == x, f, (u | 1).view(torch.float32)).half()


def _norm_rotate(x, gain, cos, sin):
    """float64, as a value next to a border of fp16 or of a code is what counts here"""
    x = x.double()
    x = x * gain.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    half = x.shape[-1] // 2
    lo, hi = x[..., :half], x[..., half:]
    return _round_once(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))


def _plain_norm(s):
    cos, sin = (t[s["pos"].long().clamp(0, MAX_POSITION - 1)].double().unsqueeze(1) for t in (s["cos"], s["sin"]))
    return [_norm_rotate(s["q"], s["g_q"], cos, sin), _norm_rotate(s["k"], s["g_k"], cos, sin)]


def _exponents(x):
    """the smallest e with max |x| <= 127 * 2^e over the last axis; infinities count as 2^16"""
    top = x.abs().amax(-1).float().clamp(max=65536.0)
    m, e = torch.frexp(top)
    return torch.where(top == 0, torch.full_like(e, E_ZERO), torch.where(m <= 127.0 / 128.0, e - 7, e - 6))


def _plain_append(s):
    q, k = _plain_norm(s)
    kc, vc = s["k_cache"], s["v_cache"]
    n_pages, Hkv, page, D = kc.shape
    slot = s["slot"].long()
    at, off = slot // page, slot % page
    start = torch.full((n_pages,), page, device=DEVICE).scatter_reduce(0, at, off, "amin")     # first new token of a page
    touched = torch.zeros(n_pages, dtype=torch.bool, device=DEVICE)
    touched[at] = True
    outs = []
    for x, codes, exps, token in ((k, kc, s["k_exp"], 2), (s["v"], vc, s["v_exp"], 3)):
        lowest = torch.full((n_pages, Hkv), -128, dtype=torch.int32, device=DEVICE)
        need = lowest.scatter_reduce(0, at[:, None].expand(-1, Hkv), _exponents(x), "amax")
        had = torch.where((touched & (start > 0))[:, None], exps.int(), lowest)
        e = torch.where(touched[:, None], torch.maximum(need, had), exps.int())
        # codes that were there: divided by the power of two that the scale grew by, halves to the even code
        shape = [1, 1, page, 1] if token == 2 else [1, 1, 1, page]
        kept = (torch.arange(page, device=DEVICE).view(shape) < start.view(-1, 1, 1, 1)) & touched.view(-1, 1, 1, 1)
        less = torch.ldexp(codes.float(), (exps.int() - e)[:, :, None, None]).round()
        codes.copy_(torch.where(kept, less, codes.float()).to(torch.int8))
        fresh = torch.ldexp(x.float(), -e[at][:, :, None]).round().clamp(-128, 127).to(torch.int8)
        if token == 2:
            codes[at, :, off, :] = fresh
        else:
            codes[at, :, :, off] = fresh
        exps.copy_(e.to(torch.int8))
        outs += [codes, exps]
    return [q, k] + outs


def _free_pages(ring, shared, taken, head, count):
    """pages that lost their last holder (shared < 0), in ascending order, behind the free ones"""
    n = ring.numel()
    gone = shared < 0
    where = torch.where(gone, (head + count + gone.long().cumsum(0) - 1) % n, torch.full_like(shared, n).long())
    ring = torch.cat([ring, ring[:1]]).scatter(0, where, torch.arange(n, device=DEVICE, dtype=torch.int32))[:n]
    return ring, torch.where(gone, torch.zeros_like(shared), shared), torch.stack([(head + taken) % n, count - taken + gone.sum()]).int()


def _plain_fork(s):
    page, length, parent, table, ring = s["page"], s["kv_len"].long(), s["parent"].long(), s["table"].long(), s["ring"]
    B, most = table.shape
    head, count = s["free"][0].long(), s["free"][1].long()
    rows, j = torch.arange(B, device=DEVICE), torch.arange(most, device=DEVICE)[None, :]
    child = parent[None, :] == rows[:, None]                                            # [request before, request after]
    n_child, first = child.sum(1), torch.where(child, rows[None, :], B).amin(1)
    of = parent.clamp(min=0)
    held, part = (length + page - 1) // page, length % page != 0
    last = table.gather(1, (held - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    joint = part & (s["shared"][last] > 0)
    copied = (parent >= 0) & part[of] & ((rows != first[of]) | joint[of])
    dst = ring[(head + copied.long().cumsum(0) - 1) % ring.numel()]
    taken = copied.sum()
    none = torch.full_like(dst, -1)
    after = torch.where(parent >= 0, length[of], 0)
    mine = table[of]
    mine = torch.where(copied[:, None] & (j == (held[of] - 1)[:, None]), dst.long()[:, None], mine)
    new_table = torch.where(j < ((after + page - 1) // page)[:, None], mine.int(), s["out"]["block_table"])
    full = j < (length // page)[:, None]
    release = part & ((n_child == 0) | joint)
    change = torch.where(full, (n_child - 1)[:, None], torch.where((j == (held - 1)[:, None]) & release[:, None], -1, 0))
    shared = torch.cat([s["shared"], s["shared"][:1] * 0]).index_add(0, torch.where(table < 0, ring.numel(), table).view(-1),
                                                                     change.view(-1).int())[:-1]
    ring, shared, free = _free_pages(ring, shared, taken, head, count)
    src = torch.where(copied, last[of].int(), none)
    dst = torch.where(copied, dst, none)
    u = copied.nonzero()[:, 0]
    for c in s["whole"]:
        c[:, dst[u].long()] = c[:, src[u].long()]
    return [after.int(), new_table, shared, src, dst, ring, free, (taken - taken).int().reshape(1)] + s["whole"]


def _plain_compact(s):
    page, length, stay, table, ring = s["page"], s["kv_len"].long(), s["stay"].long(), s["table"].long(), s["ring"]
    B, most = table.shape
    head, count = s["free"][0].long(), s["free"][1].long()
    cu = s["cu_keep"].long()
    n = cu[1:] - cu[:-1]
    stay = torch.minimum(stay, length)
    after = stay + n
    held, total = (length + page - 1) // page, (after + page - 1) // page
    j = torch.arange(most, device=DEVICE)[None, :]
    last = table.gather(1, (total - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    joint = (n == 0) & (after < length) & (after % page != 0) & (s["shared"][last] > 0)    # would be written into, but is not its own
    same = torch.where(n > 0, stay // page, torch.where(joint, total - 1, total))         # pages that stay
    need = total - same
    at = need.cumsum(0) - need
    fresh = (j >= same[:, None]) & (j < total[:, None])
    got = ring[(head + at[:, None] + j - same[:, None]) % ring.numel()]
    new_table = torch.where(fresh, got, torch.where(j < total[:, None], table.int(), s["out"]["block_table"]))
    gone = (j >= same[:, None]) & (j < held[:, None])
    shared = torch.cat([s["shared"], s["shared"][:1] * 0]).index_add(0, torch.where(table < 0, ring.numel(), table).view(-1),
                                                                     -gone.view(-1).int())[:-1]
    new_ring, shared, free = _free_pages(ring, shared, need.sum(), head, count)
    # the new pages, and the tokens that go into them
    b, e = fresh.nonzero(as_tuple=True)
    if b.numel():
        to = new_table[b, e].long()
        i = e[:, None] * page + torch.arange(page, device=DEVICE)[None, :]
        there = i < after[b][:, None]
        listed_at = (cu[b][:, None] + i - stay[b][:, None]).clamp(0, max(0, s["keep"].numel() - 1))
        old = torch.where(i < stay[b][:, None], i, s["keep"].long()[listed_at] if s["keep"].numel() else i)
        old = torch.where(there, old, 0)
        src, off = table[b[:, None], old // page].clamp(min=0), old % page
        for kc, vc, ke, ve in s["caches"]:
            for codes, exps, turn in ((kc, ke, False), (vc, ve, True)):
                x = codes[src, :, :, off] if turn else codes[src, :, off, :]               # [pages, tokens, heads, D]
                had = torch.where(there[:, :, None], exps[src].int(), -128)
                new = had.amax(1, keepdim=True)
                x = torch.ldexp(x.float(), (had - new)[..., None]).round()
                x = torch.where(there[:, :, None, None], x, 0.0).to(torch.int8)
                codes[to] = x.permute(0, 2, 3, 1) if turn else x.permute(0, 2, 1, 3)
                exps[to] = new[:, 0].to(torch.int8)
    return [after.int(), new_table, shared, new_ring, free, (after[0] * 0).int().reshape(1)] + s["whole"]


def run(s):
    if not own:
        return {"score": _plain_score, "norm": _plain_norm, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[s["kind"]](s)
    from paper_2312_05693_amd import binding as agq
    if s["kind"] == "score":
        got = agq.logprobs(s["logits"], s["tokens"], n_top=s["case"]["n_top"])
        return [t for t in got if t is not None]
    if s["kind"] == "norm":
        return list(agq.qk_norm_rope(s["q"], s["k"], s["g_q"], s["g_k"], EPS, s["pos"], s["cos"], s["sin"]))
    if s["kind"] == "append":
        q, k = agq.kv_append_norm(s["k"], s["v"], s["slot"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["g_k"], EPS, q=s["q"],
                                  g_q=s["g_q"], pos=s["pos"], rope_cos=s["cos"], rope_sin=s["sin"])
        return [q, k, s["k_cache"], s["k_exp"], s["v_cache"], s["v_exp"]]
    if s["kind"] == "fork":
        f = agq.kv_fork(s["kv_len"], s["parent"], s["table"], s["page"], s["shared"], s["ring"], s["free"], out=s["step"])
        agq.kv_copy_pages(s["layers"], f.copy_src, f.copy_dst)
        return [f.kv_len, f.block_table, f.shared, f.copy_src, f.copy_dst, s["ring"], f.free_state, f.status] + s["whole"]
    c = agq.kv_compact(s["kv_len"], s["stay"], s["cu_keep"], s["keep"], s["table"], s["page"], s["shared"], s["ring"], s["free"], out=s["step"])
    agq.kv_move(s["layers"], c.moves, s["table"], s["stay"], s["cu_keep"], s["keep"])
    return [c.kv_len, c.block_table, c.shared, s["ring"], c.free_state, c.status] + s["whole"]


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_score(s):
    n, logp, entropy, index, best = s["case"]["n_top"], [], [], [], []
    for t0 in range(0, s["logits"].shape[0], 256):
        x = s["logits"][t0:t0 + 256].double()
        every = x - torch.logsumexp(x, 1, keepdim=True)
        logp.append(every.gather(1, s["tokens"][t0:t0 + 256].long()[:, None])[:, 0])
        entropy.append(torch.special.entr(torch.exp(every)).sum(1))
        if n:
            order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :n]
            index.append(order.int())
            best.append(every.gather(1, order))
    out = [torch.cat(logp), torch.cat(entropy)]
    return out + ([torch.cat(index), torch.cat(best)] if n else [])


def _exact_heads(x, gain, cos, sin, pos):
    """(values in float64, the same rounded to fp16)"""
    x, gain = x.cpu().numpy().astype(np.float64), gain.cpu().numpy().astype(np.float64)
    y = x / np.sqrt(np.square(x).sum(-1, keepdims=True) / x.shape[-1] + EPS) * gain
    c, n = (t.cpu().numpy().astype(np.float64)[pos][:, None, :] for t in (cos, sin))
    a, b = np.split(y, 2, -1)
    y = np.concatenate([a * c - b * n, b * c + a * n], -1)
    return y, y.astype(np.float16)


def _exact_append(s, kr):
    slot = s["slot"].cpu().numpy()
    n_pages, Hkv, page, D = s["k_cache"].shape
    run_at, run_to, res = {}, {}, []
    for t, sl in enumerate(slot):
        run_at.setdefault(int(sl) // page, t)
        run_to[int(sl) // page] = t + 1
    for x, name, turn in ((kr, "k", False), (s["v"].cpu().numpy(), "v", True)):
        codes, exps = s[name + "_cache"].cpu().numpy().copy(), s[name + "_exp"].cpu().numpy().astype(np.int64)
        for p, t0 in run_at.items():
            t1, o0 = run_to[p], int(slot[t0]) % page
            rows = x[t0:t1].astype(np.float64).transpose(1, 0, 2)              # [Hkv, tokens, D]
            top = np.minimum(np.abs(rows).max((1, 2)), 65536.0)
            need = np.full(Hkv, E_ZERO)
            for e in range(10, E_ZERO - 1, -1):
                need[top <= 127.0 * 2.0 ** e] = e
            e = np.maximum(need, exps[p]) if o0 else need
            page_codes = codes[p].transpose(0, 2, 1) if turn else codes[p]     # [Hkv, page, D], a view
            page_codes[:, :o0] = np.rint(page_codes[:, :o0] * 2.0 ** (exps[p] - e)[:, None, None])
            page_codes[:, o0:o0 + t1 - t0] = np.clip(np.rint(rows * 2.0 ** -e[:, None, None]), -128, 127)
            exps[p] = e
        res += [torch.from_numpy(codes).to(DEVICE), torch.from_numpy(exps.astype(np.int8)).to(DEVICE)]
    return res


def _host(s, *names):
    return [s[n].cpu().numpy().astype(np.int64) for n in names]


def _give_back(lost, ring, shared, head, count, took):
    """holders who let go of pages, and the pages that nobody holds then"""
    for p, n in lost.items():
        shared[p] += n
    back = sorted(p for p in lost if shared[p] < 0)
    for i, p in enumerate(back):
        ring[(head + count + i) % len(ring)] = p
        shared[p] = 0
    return [(head + took) % len(ring), count - took + len(back)]


def _exact_fork(s):
    page = s["page"]
    length, parent, table, shared, ring, (head, count) = _host(s, "kv_len", "parent", "table", "shared", "ring", "free")
    B, free = len(length), [int(ring[(int(head) + i) % len(ring)]) for i in range(int(count))]
    new_table, was, lost = s["out"]["block_table"].cpu().numpy().astype(np.int64), shared.copy(), {}
    src, dst, lens, seen, took = [-1] * B, [-1] * B, [], set(), 0
    for b, p in enumerate(parent.tolist()):
        lens.append(int(length[p]) if p >= 0 else 0)
        if p < 0:
            continue
        held = -(-lens[b] // page)
        new_table[b, :held] = table[p, :held]
        for x in table[p, :lens[b] // page].tolist():
            lost[x] = lost.get(x, 0) + 1
        if lens[b] % page:
            x = int(table[p, held - 1])
            if p in seen or was[x] > 0:
                src[b], dst[b] = x, free[took]
                new_table[b, held - 1] = free[took]
                took += 1
            else:
                lost[x] = lost.get(x, 0) + 1
        seen.add(p)
    for b in range(B):                                                          # what every request held before
        for x in table[b, :-(-int(length[b]) // page)].tolist():
            lost[x] = lost.get(x, 0) - 1
    state = _give_back(lost, ring, shared, int(head), int(count), took)
    caches = []
    for c in s["whole"]:
        c = c.clone()
        for x, y in zip(src, dst):
            if y >= 0:
                c[:, y] = c[:, x]
        caches.append(c)
    return [_int32(a) for a in (lens, new_table, shared, src, dst, ring, state, [0])] + caches


def _exact_compact(s):
    page = s["page"]
    length, stay, cu, keep, table, shared, ring, (head, count) = _host(s, "kv_len", "stay", "cu_keep", "keep", "table", "shared", "ring", "free")
    B, free = len(length), [int(ring[(int(head) + i) % len(ring)]) for i in range(int(count))]
    new_table, was, lost, lens, took, jobs = s["out"]["block_table"].cpu().numpy().astype(np.int64), shared.copy(), {}, [], 0, []
    for b in range(B):
        tokens = np.concatenate([np.arange(min(stay[b], length[b])), keep[cu[b]:cu[b + 1]]]).astype(np.int64)
        n, held, listed_any = len(tokens), -(-int(length[b]) // page), cu[b + 1] > cu[b]
        lens.append(n)
        for j in range(-(-n // page)):
            here, full = tokens[j * page:(j + 1) * page], n >= (j + 1) * page
            same = (j + 1) * page <= stay[b] if listed_any else n == length[b] or full or was[table[b, j]] == 0
            new_table[b, j] = table[b, j] if same else free[took]
            if not same:
                jobs.append((free[took], table[b, here // page], here % page))
                took += 1
                lost[int(table[b, j])] = lost.get(int(table[b, j]), 0) - (j < held)
        for j in range(-(-n // page), held):
            lost[int(table[b, j])] = lost.get(int(table[b, j]), 0) - 1
    state = _give_back(lost, ring, shared, int(head), int(count), took)
    caches = []
    for kc, vc, ke, ve in s["caches"]:
        for c, e, turn in ((kc, ke, False), (vc, ve, True)):
            c, e = c.cpu().numpy().copy(), e.cpu().numpy().copy()
            rows = c.transpose(0, 1, 3, 2) if turn else c                       # [pages, heads, tokens, D], a view
            done = []
            for to, p, off in jobs:
                had = e[p].astype(np.int64)                                     # [tokens, heads]
                top = had.max(0)
                done.append((to, np.rint(rows[p, :, off].astype(np.float64) * 2.0 ** (had - top)[:, :, None]), top))
            for to, x, top in done:
                rows[to] = 0
                rows[to, :, :len(x)] = x.transpose(1, 0, 2)
                e[to] = top
            caches += [torch.from_numpy(c).to(DEVICE), torch.from_numpy(e).to(DEVICE)]
    caches = [torch.stack(caches[k::4]) for k in (0, 2, 1, 3)]                  # keys, values, exponents of keys, exponents of values
    return [_int32(a) for a in (lens, new_table, shared, ring, state, [0])] + caches


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "score":
        return _exact_score(s)
    if s["kind"] == "fork":
        return _exact_fork(s)
    if s["kind"] == "compact":
        return _exact_compact(s)
    pos = s["pos"].cpu().numpy()
    (q, _), (k, kr) = (_exact_heads(s[n], s["g_" + n], s["cos"], s["sin"], pos) for n in ("q", "k"))
    out = [torch.from_numpy(q).to(DEVICE), torch.from_numpy(k).to(DEVICE)]
    return out if s["kind"] == "norm" else out + _exact_append(s, kr)
