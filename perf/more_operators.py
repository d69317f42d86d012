"""What stands around a decoder layer's attention, as measurable cases: the norm and the rotation by position that its
queries and keys get on their way out of the projection and into the cache, the weights that its keys receive, and the
cache that is cut down to the rows which received most.

The skip KV-cache (Section 4.3) drops the rows of skipped tokens after the prefill; these operators go on from there.
Every key sums the attention weights it receives, in the prefill and in every step after it, and a sequence whose rows
exceed its budget keeps those with the largest sums, each key/value head its own.  Sizes: a LLaMA-3-8B layer (32 query
heads, 8 key/value heads, 128 columns a head), LLaVA sequences of 576 visual + 40 text tokens, high-resolution sequences of
5 x 576 visual + 64 text tokens, the repository's small layer, and generic ones.

  listed()   the fixed cases            draw(rng)  one more of the same ranges
  prepare()  what a program holds       run()      one pass over it
  work()     bytes and operations       exact()    the outputs in 64 bits
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
LOG2E = 1.4426950408889634


# ---- the cases -------------------------------------------------------------------------------------
def _case(name, **c):
    return dict(c, name=name) if name else c


def rope(name, *, seqs, tokens, use="serve", axes=1, axis_order="sections", norm=True, pairs=False, far=0, rot=0, ragged=0,
         heads=32, kv_heads=8, dim=128):
    """q and k of `seqs` sequences of `tokens` tokens, from position `far` on.  use: "serve" puts k and v into the rows of a cache,
    "train" goes forward and back.  rot: columns of a head that are rotated (0: all).  pairs: neighbouring columns are rotated
    together, otherwise those of the two halves."""
    return _case(name, kind="rope", seqs=seqs, tokens=tokens, use=use, axes=axes, axis_order=axis_order, norm=norm, pairs=pairs,
                 far=far, rot=rot or dim, ragged=ragged, heads=heads, kv_heads=kv_heads, dim=dim)


def weights(name, *, seqs, tokens, past=0, last=0, ragged=0, heads=32, kv_heads=8, dim=128, causal=True):
    """What the keys receive from `seqs` packed sequences of `tokens` queries after `past` cached tokens; last: from the
    last so many queries of a sequence only (0: all)."""
    return _case(name, kind="weights", seqs=seqs, tokens=tokens, past=past, last=last, ragged=ragged, heads=heads, kv_heads=kv_heads,
                 dim=dim, causal=causal)


def step(name, *, seqs, shared, prefix, suffix, ragged=0, heads=32, kv_heads=8, dim=128):
    """One new token for each of `seqs` sequences, and what the cache's rows receive from it.  `shared` sequences at a time have the
    same cached beginning of `prefix` tokens; each has up to `suffix` further tokens of its own."""
    return _case(name, kind="step", seqs=seqs, shared=shared, prefix=prefix, suffix=suffix, ragged=ragged, heads=heads,
                 kv_heads=kv_heads, dim=dim)


def evict(name, *, seqs, rows, keep, first=4, recent=0, packed=True, ragged=0, kv_heads=8, dim=128):
    """`seqs` caches of `rows` rows cut down to `keep` of them, of which the `first` and the `recent` ones stay whatever they
    received.  packed: one after the other, or each with a capacity of its own."""
    return _case(name, kind="evict", seqs=seqs, rows=rows, keep=keep, first=first, recent=recent, packed=packed, ragged=ragged,
                 kv_heads=kv_heads, dim=dim)


def listed():
    return [
        # a decode step of 64 sequences at far positions: latency
        rope("rope_decode_b64", seqs=64, tokens=1, far=100000),
        # prefill of 4 high-resolution images whose patches have a time, a row and a column, into the cache
        rope("rope_images_b4", seqs=4, tokens=2944, axes=3, norm=False),
        # a training step of 16 sequences (the repository's default workload), forward and back
        rope("rope_train_b16", seqs=16, tokens=616, use="train"),
        # the repository's small layer
        weights("weights_small_layer", seqs=1, tokens=80, heads=4, kv_heads=4, dim=64),
        # prefill of a batch of 16 requests of different length
        weights("weights_b16", seqs=16, tokens=616, ragged=5),
        # one long document, judged by its last 64 tokens
        weights("weights_window", seqs=1, tokens=32768, last=64),
        # one long document, judged by all of its tokens
        weights("weights_long", seqs=1, tokens=16384),
        # one decode step of 8 sequences, each with its own image of 144 retained + 40 text tokens
        step("step_b8", seqs=8, shared=1, prefix=184, suffix=64),
        # one decode step of 64 answers, 32 of them about each of two long inputs
        step("step_shared_b64", seqs=64, shared=32, prefix=5795, suffix=256, ragged=9),
        # one decode step of 4 sequences with long caches of their own
        step("step_long_b4", seqs=4, shared=1, prefix=32768, suffix=512, ragged=8),
        # the caches of 64 answers, full: half of the budget is recent
        evict("evict_own_b64", seqs=64, rows=1000, keep=500, recent=250, packed=False, ragged=6),
        # after the prefill of 4 long documents
        evict("evict_long_b4", seqs=4, rows=32768, keep=8000, recent=4000, ragged=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 32), (16, 16), (16, 2), (12, 4), (28, 4), (8, 1), (6, 6)])
    dim = rng.choice([128, 128, 128, 64, 64, 80, 96, 40, 72])
    ragged = rng.choice([0, rng.randint(1, 10**6), rng.randint(1, 10**6)])
    kind = rng.choice(["rope", "weights", "append", "step", "evict"])
    shape = dict(ragged=ragged, heads=heads, kv_heads=kv_heads, dim=dim)
    if kind == "rope":
        tokens = _log(rng, 1, 8192)
        return rope(None, seqs=max(1, min(_log(rng, 1, 64), 16384 // tokens)), tokens=tokens, use=rng.choice(["serve", "train"]),
                    axes=rng.choice([1, 1, 2, 3]), axis_order=rng.choice(["sections", "turns"]), norm=rng.random() < 0.6,
                    pairs=rng.random() < 0.3, far=rng.choice([0, _log(rng, 1, 10**6)]), rot=rng.choice([dim, dim, dim // 16 * 8]), **shape)
    if kind == "weights":
        tokens = _log(rng, 1, 8192)
        return weights(None, seqs=max(1, min(_log(rng, 1, 32), 12288 // tokens)), tokens=tokens,
                       last=rng.choice([0, 0, _log(rng, 1, 128)]), causal=rng.random() < 0.8, **shape)
    if kind == "append":
        past = _log(rng, 100, 16384)
        return weights(None, seqs=max(1, min(_log(rng, 1, 16), 32768 // past)), tokens=_log(rng, 1, 500), past=past,
                       last=rng.choice([0, _log(rng, 1, 128)]), **shape)
    if kind == "step":
        prefix, shared = _log(rng, 16, 32768), _log(rng, 1, 64)
        groups = max(1, min(_log(rng, 1, 32), 131072 // prefix))
        return step(None, seqs=min(128, shared * groups), shared=shared, prefix=prefix, suffix=_log(rng, 1, 512), **shape)
    rows = _log(rng, 16, 65536)
    keep = max(1, _log(rng, 1, rows))
    return evict(None, seqs=max(1, min(_log(rng, 1, 64), 131072 // rows)), rows=rows, keep=keep, first=rng.choice([0, 1, 4, 16]),
                 recent=rng.choice([0, keep // 2, rng.randint(0, keep)]), packed=rng.random() < 0.5, ragged=ragged, kv_heads=kv_heads, dim=dim)


# ---- sizes that follow from a case -------------------------------------------------------------------
def _sizes(n, full, ragged, salt):
    if not ragged or not full:
        return [full] * n
    r = random.Random(ragged * 1000 + salt)
    return [r.randint(max(1, full // 5), full) for _ in range(n)]


def _offsets(sizes):
    out = [0]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def _prompt_sizes(c):
    """Queries and keys of every sequence, and how many of the queries count."""
    new, past = _sizes(c["seqs"], c["tokens"], c["ragged"], 1), _sizes(c["seqs"], c["past"], c["ragged"], 2)
    return new, [a + b for a, b in zip(new, past)], [min(a, c["last"]) if c["last"] else a for a in new]


def _step_sizes(c):
    """Sequences of every group, its cached tokens, and every sequence's own tokens."""
    groups = -(-c["seqs"] // c["shared"])
    members = [min(c["shared"], c["seqs"] - i * c["shared"]) for i in range(groups)]
    return members, _sizes(groups, c["prefix"], c["ragged"], 3), _sizes(c["seqs"], c["suffix"], c["ragged"], 4)


def work(c):
    K, D = c["kv_heads"], c["dim"]
    if c["kind"] == "evict":
        rows = _sizes(c["seqs"], c["rows"], c["ragged"], 5)
        kept = sum(min(n, c["keep"]) for n in rows)
        # weights; kept keys and values in and out, their weights and numbers out
        return {"bytes": K * (4 * sum(rows) + kept * (8 * D + 8)), "flops": 0}
    H = c["heads"]
    if c["kind"] == "rope":
        T = sum(_sizes(c["seqs"], c["tokens"], c["ragged"], 1))
        once = 4 * D * T * (H + (2 if c["use"] == "serve" else 1) * K) + 4 * T * c["axes"]
        # back: the gradients in and out, and with a norm q and k again
        back = (4 + (2 if c["norm"] else 0)) * D * T * (H + K) if c["use"] == "train" else 0
        return {"bytes": once + back, "flops": (20 if back else 8) * D * T * (H + K)}
    if c["kind"] == "step":
        members, prefix, suffix = _step_sizes(c)
        seen, rows = sum(m * p for m, p in zip(members, prefix)) + sum(suffix), sum(prefix) + sum(suffix)
        return {"bytes": rows * K * (4 * D + 4) + 4 * D * H * c["seqs"], "flops": 4 * D * H * seen}
    new, keys, count = _prompt_sizes(c)
    pairs = sum(m * k - (m * (m - 1) // 2 if c["causal"] else 0) for m, k in zip(count, keys))
    # counted queries and their log-sum-exps, keys, weights
    return {"bytes": (2 * D + 4) * (H * sum(count) + K * sum(keys)), "flops": 2 * D * H * pairs}


# ---- inputs --------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _axes_of(c):
    """The position axis of every rotated pair of columns."""
    n, a = c["rot"] // 2, c["axes"]
    if c["axis_order"] == "turns":
        return [j % a for j in range(n)]
    first = n // 4 if a > 1 else n                       # time has fewer than height and width
    return [0 if j < first else 1 + (j - first) * (a - 1) // (n - first) for j in range(n)]


def _positions(c, sizes):
    """[axes, T]: the place in its sequence; with several axes patches of images of 24 columns a row have a time, a row and a column."""
    out = []
    for n in sizes:
        t = torch.arange(n, device="cuda")
        out.append(torch.stack([t if c["axes"] == 1 else t // 576, t // 24 % 24, t % 24][:c["axes"]]))
    return (torch.cat(out, 1) + c["far"]).to(torch.int32).contiguous()


def _prepare_rope(c, gen):
    H, K, D, sizes = c["heads"], c["kv_heads"], c["dim"], _sizes(c["seqs"], c["tokens"], c["ragged"], 1)
    T = sum(sizes)
    qkv = _normal(gen, T, H + 2 * K, D)                  # the projection's output, one row a token
    freq = 500000.0 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64) * 2 / c["rot"])
    s = dict(kind="rope", use=c["use"], norm=c["norm"], pairs=c["pairs"], rot=c["rot"], axis=_axes_of(c), pos=_positions(c, sizes),
             inv_freq=freq.float().cuda(), q=qkv[:, :H], k=qkv[:, H:H + K], v=qkv[:, H + K:], gain_q=None, gain_k=None,
             q_out=torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda"))
    if c["norm"]:
        s.update(gain_q=(1 + 0.2 * _normal(gen, D).float()).to(torch.bfloat16), gain_k=(1 + 0.2 * _normal(gen, D).float()).to(torch.bfloat16))
    if c["use"] == "serve":
        # every sequence's new rows come after some that are there, in a cache [key or value][head][row][column]
        before = [5 + i % 3 for i in range(len(sizes))]
        cap = max(sizes) + 8
        cache = _normal(gen, 2, K, len(sizes) * cap, D)
        row = torch.cat([i * cap + before[i] + torch.arange(n, device="cuda") for i, n in enumerate(sizes)]).to(torch.int32)
        s.update(cache=cache, row=row)
    else:
        s.update(k_out=torch.empty(T, K, D, dtype=torch.bfloat16, device="cuda"), grad_q_out=_normal(gen, T, H, D),
                 grad_k_out=_normal(gen, T, K, D), grad_qkv=torch.zeros(T, H + 2 * K, D, dtype=torch.bfloat16, device="cuda"),
                 d_gain_q=torch.zeros(D, device="cuda"), d_gain_k=torch.zeros(D, device="cuda"))
    return s


def _prepare_weights(c, gen):
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    new, keys, count = _prompt_sizes(c)
    T, Tk, g = sum(new), sum(keys), H // K
    if c["past"]:
        q, k = _normal(gen, T, H, D), _normal(gen, K, Tk, D).transpose(0, 1)
    else:
        qkv = _normal(gen, T, H + 2 * K, D)
        q, k = qkv[:, :H], qkv[:, H:H + K]
    # what the attention saved: the logarithm (base 2) of every row's sum of weights, [query head][token]
    saved = torch.zeros(H * T * 4 + 256, dtype=torch.uint8, device="cuda")
    lse = saved[:H * T * 4].view(torch.float32).view(H, T)
    qo, ko = _offsets(new), _offsets(keys)
    for b, (nq, nk, m) in enumerate(zip(new, keys, count)):
        kb = k[ko[b]:ko[b + 1]].float().permute(1, 2, 0)                     # [K, D, nk]
        for i in range(nq - m, nq, 2048):
            e = min(nq, i + 2048)
            see = torch.arange(nk, device="cuda") <= torch.arange(i, e, device="cuda")[:, None] + (nk - nq if c["causal"] else nk)
            for h in range(H):
                x = (q[qo[b] + i:qo[b] + e, h].float() @ kb[h // g]).mul_(LOG2E / math.sqrt(D)).masked_fill_(~see, -math.inf)
                top = x.amax(-1, keepdim=True)
                lse[h, qo[b] + i:qo[b] + e] = torch.log2(torch.exp2(x - top).sum(-1)) + top[:, 0]
    return dict(kind="weights", q=q, k=k, saved=saved, causal=c["causal"], last=c["last"], scale=1.0 / math.sqrt(D), seg_q=_ints(qo),
                seg_k=_ints(ko), most_q=max(count), most_k=max(keys), weights=torch.zeros(K, Tk, device="cuda"))


def _prepare_step(c, gen):
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    members, prefix, suffix = _step_sizes(c)
    # a compacted cache keeps its capacity: [key/value head][token][column], of which the first rows are in use
    cap, own_cap, n = sum(prefix) + 64, c["suffix"] + 8, c["seqs"]
    cache, own_cache = _normal(gen, 2, K, cap, D), _normal(gen, 2, n, K, own_cap, D)
    return dict(kind="step", scale=1.0 / math.sqrt(D), q=_normal(gen, n, H, D), out=torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"),
                prefix_k=cache[0].transpose(0, 1), prefix_v=cache[1].transpose(0, 1),
                suffix_k=own_cache[0].transpose(1, 2), suffix_v=own_cache[1].transpose(1, 2),
                prefix_seg=_ints(_offsets(prefix)), group_off=_ints(_offsets(members)), suffix_len=_ints(suffix),
                prefix_weights=torch.zeros(K, cap, device="cuda"), suffix_weights=torch.zeros(n, K, own_cap, device="cuda"),
                longest=max(prefix), members=max(members))


def _prepare_evict(c, gen):
    K, D, n = c["kv_heads"], c["dim"], c["seqs"]
    rows = _sizes(n, c["rows"], c["ragged"], 5)
    s = dict(kind="evict", n_keep=c["keep"], first=c["first"], recent=c["recent"], packed=c["packed"], most=max(rows))
    # sums of weights: a few rows hold most of it, some received nothing at all
    if c["packed"]:
        T, out = sum(rows), sum(min(x, c["keep"]) for x in rows)
        cache, new, shape, new_shape = _normal(gen, 2, K, T, D), (2, K, out, D), (K, T), (K, out)
        s.update(seg=_ints(_offsets(rows)), seg_out=torch.zeros(n + 1, dtype=torch.int32, device="cuda"))
    else:
        cap = c["rows"] + 8
        cache, new, shape, new_shape = _normal(gen, 2, n, K, cap, D), (2, n, K, cap, D), (n, K, cap), (n, K, cap)
        s.update(seg=_ints(rows), seg_out=torch.zeros(n, dtype=torch.int32, device="cuda"))
    w = torch.exp(2.0 * torch.randn(shape, generator=gen, device="cuda"))
    w = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.1, torch.zeros_like(w), w)
    fresh = torch.zeros(new, dtype=torch.bfloat16, device="cuda")
    s.update(k=cache[0].transpose(-3, -2), v=cache[1].transpose(-3, -2), weights=w, k_out=fresh[0].transpose(-3, -2),
             v_out=fresh[1].transpose(-3, -2), weights_out=torch.zeros(new_shape, device="cuda"),
             keep=torch.zeros(new_shape, dtype=torch.int32, device="cuda"))
    return s


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return dict(rope=_prepare_rope, weights=_prepare_weights, step=_prepare_step, evict=_prepare_evict)[c["kind"]](c, gen)


# ---- one pass through the framework ----------------------------------------------------------------------
def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _own_rope(s):
    from paper_2503_21817_amd import binding as B
    (T, H, D), K = s["q"].shape, s["k"].shape[1]
    if "axis_bytes" not in s:
        s["axis_bytes"] = bytes(s["axis"]) if s["pos"].shape[0] > 1 else None
    flags = (B.FLAG_QK_NORM if s["norm"] else 0) | (B.FLAG_ROPE_PAIRS if s["pairs"] else 0)
    norm = dict(gain_q=s["gain_q"], gain_k=s["gain_k"], eps=EPS) if s["norm"] else {}
    if s["use"] == "serve":
        B.skipffn_qk_rope_forward(s["q"], s["k"], s["q_out"], s["cache"][0].transpose(0, 1), s["pos"], s["inv_freq"], axis=s["axis_bytes"],
                                  v=s["v"], v_out=s["cache"][1].transpose(0, 1), row=s["row"], flags=flags, **norm)
        return s["q_out"], s["cache"]
    if "workspace" not in s:
        s["workspace"] = _bytes(B.skipffn_qk_rope_backward_workspace_bytes(T, H, K, D))
    B.skipffn_qk_rope_forward(s["q"], s["k"], s["q_out"], s["k_out"], s["pos"], s["inv_freq"], axis=s["axis_bytes"], flags=flags, **norm)
    gq, gk = s["grad_qkv"][:, :H], s["grad_qkv"][:, H:H + K]
    more = dict(norm, q=s["q"], k=s["k"], d_gain_q=s["d_gain_q"], d_gain_k=s["d_gain_k"]) if s["norm"] else {}
    B.skipffn_qk_rope_backward(s["grad_q_out"], s["grad_k_out"], gq, gk, s["pos"], s["inv_freq"], axis=s["axis_bytes"], flags=flags,
                               workspace=s["workspace"], **more)
    return (s["q_out"], s["k_out"], s["grad_qkv"]) + ((s["d_gain_q"], s["d_gain_k"]) if s["norm"] else ())


def _own_weights(s):
    from paper_2503_21817_amd import binding as B
    (T, H, D), (Tk, K, _), n = s["q"].shape, s["k"].shape, s["seg_q"].numel() - 1
    last = s["last"] or None
    if "workspace" not in s:
        s["workspace"] = _bytes(B.skipffn_attn_key_weights_workspace_bytes(T, Tk, n, H, K, D, last))
    B.skipffn_attn_key_weights(s["q"], s["k"], s["seg_q"], s["seg_k"], s["saved"], s["weights"], causal=s["causal"], scale=s["scale"],
                               last=last, workspace=s["workspace"])
    return s["weights"]


def _own_step(s):
    from paper_2503_21817_amd import binding as B
    (n, H, D), (Tp, K, _) = s["q"].shape, s["prefix_k"].shape
    if "workspace" not in s:
        s["workspace"] = _bytes(B.skipffn_attn_decode_weights_workspace_bytes(n, s["group_off"].numel() - 1, H, K, D, Tp,
                                                                              s["suffix_k"].shape[1], s["members"]))
    B.skipffn_attn_decode_weights(s["q"], s["prefix_k"], s["prefix_v"], s["prefix_seg"], s["group_off"], s["suffix_k"], s["suffix_v"],
                                  s["suffix_len"], s["out"], s["prefix_weights"], s["suffix_weights"], most_shared=s["members"],
                                  scale=s["scale"], workspace=s["workspace"])
    return s["out"], s["prefix_weights"], s["suffix_weights"]


def _own_evict(s):
    from paper_2503_21817_amd import binding as B
    B.skipffn_kv_evict(s["k"], s["v"], s["weights"], s["seg"], s["n_keep"], s["k_out"], s["v_out"], s["weights_out"], s["keep"],
                       s["seg_out"], first=s["first"], recent=s["recent"])
    return s["k_out"], s["v_out"], s["weights_out"], s["keep"], s["seg_out"]


# ---- one pass in elementary operations ---------------------------------------------------------------------
def _columns(s, D):
    """The first and the second column of every rotated pair."""
    j = torch.arange(s["rot"] // 2, device="cuda")
    return (2 * j, 2 * j + 1) if s["pairs"] else (j, j + s["rot"] // 2)


def _turn(x, s, sign):
    """Rotates the pairs of x [T, heads, D] in float32; the angles, which may be of far positions, are taken in 64 bits."""
    a, b = _columns(s, x.shape[-1])
    at = s["pos"].double()[torch.tensor(s["axis"], device="cuda")].T * s["inv_freq"].double()       # [T, rot / 2]
    at = torch.remainder(at, 2 * math.pi).float()[:, None]
    cos, sin = torch.cos(at), sign * torch.sin(at)
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., a] * sin + x[..., b] * cos
    return y


def _plain_rope(s):
    (T, H, D), K = s["q"].shape, s["k"].shape[1]

    def forward(x, gain):
        x = x.float()
        if s["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
        return _turn(x, s, 1.0).to(torch.bfloat16)

    def back(x, gain, grad):
        g = _turn(grad.float(), s, -1.0)
        if not s["norm"]:
            return g.to(torch.bfloat16), None
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        d_gain = (g * (x * r)).sum((0, 1), dtype=torch.float64).float()
        g = g * gain.float()
        return (r * (g - x * (r * r * (g * x).mean(-1, keepdim=True)))).to(torch.bfloat16), d_gain

    s["q_out"].copy_(forward(s["q"], s["gain_q"]))
    k = forward(s["k"], s["gain_k"])
    if s["use"] == "serve":
        at = s["row"].long()
        s["cache"][0][:, at] = k.transpose(0, 1)
        s["cache"][1][:, at] = s["v"].transpose(0, 1)
        return s["q_out"], s["cache"]
    s["k_out"].copy_(k)
    s["grad_qkv"][:, :H], dgq = back(s["q"], s["gain_q"], s["grad_q_out"])
    s["grad_qkv"][:, H:H + K], dgk = back(s["k"], s["gain_k"], s["grad_k_out"])
    return (s["q_out"], s["k_out"], s["grad_qkv"]) + ((dgq, dgk) if s["norm"] else ())


def _padded(x, first, end, most):
    """Rows first .. end of packed sequences [T, heads, D] as [sequence, head, most, D] in float32 (rows past a sequence's end repeat
    one), and which of them are real."""
    at = torch.arange(most, device=x.device)
    real = at < (end - first)[:, None]
    rows = (first[:, None] + at).clamp(max=x.shape[0] - 1).long()
    return x[rows].float().transpose(1, 2), real, rows


def _plain_weights(s):
    (T, H, D), (Tk, K, _) = s["q"].shape, s["k"].shape
    seg_q, seg_k, g, mq, mk = s["seg_q"], s["seg_k"], H // K, s["most_q"], s["most_k"]
    n = seg_q.numel() - 1
    begin = torch.maximum(seg_q[:-1], seg_q[1:] - s["last"]) if s["last"] else seg_q[:-1]
    q, real_q, rows_q = _padded(s["q"], begin, seg_q[1:], mq)
    k, real_k, rows_k = _padded(s["k"], seg_k[:-1], seg_k[1:], mk)
    lse = s["saved"][:H * T * 4].view(torch.float32).view(H, T)[:, rows_q].transpose(0, 1)          # [sequence, H, mq]
    sees = real_q[:, :, None] & real_k[:, None, :]
    if s["causal"]:
        # a sequence's last query sees all its keys, the one before it all but one
        i, j = torch.arange(mq, device=q.device), torch.arange(mk, device=q.device)
        ahead = (seg_k[1:] - seg_k[:-1]) - (seg_q[1:] - begin)
        sees &= j[None, None, :] <= i[None, :, None] + ahead[:, None, None]
    per = max(1, (1 << 30) // (n * g * mq * mk))          # key/value heads at a time
    real_rows = rows_k[real_k]
    for h in range(0, K, per):
        m = min(per, K - h)
        x = torch.matmul(q[:, h * g:(h + m) * g].reshape(n, m, g * mq, D), k[:, h:h + m].transpose(2, 3)).view(n, m, g, mq, mk)
        x.mul_(s["scale"] * LOG2E).sub_(lse[:, h * g:(h + m) * g].reshape(n, m, g, mq, 1)).exp2_()
        x.masked_fill_(~sees[:, None, None], 0.0)
        w = x.sum((2, 3))                                # [sequence, heads, mk]
        s["weights"][h:h + m, real_rows] = w.transpose(0, 1)[:, real_k]
    return s["weights"]


def _plain_step(s):
    (n, H, D), K = s["q"].shape, s["prefix_k"].shape[1]
    off, seg, m, g = s["group_off"], s["prefix_seg"], s["members"], H // K
    q, real_q, _ = _padded(s["q"], off[:-1], off[1:], m)                  # [group, H, member, D]
    G = q.shape[0]
    q = q.reshape(G, K, g * m, D)
    k, real, rows = _padded(s["prefix_k"], seg[:-1], seg[1:], s["longest"])
    v, _, _ = _padded(s["prefix_v"], seg[:-1], seg[1:], s["longest"])
    p = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    p.masked_fill_(~real[:, None, None, :], float("-inf"))
    qs = s["q"].float().view(n, K, g, D)
    ks, vs = s["suffix_k"].float().transpose(1, 2), s["suffix_v"].float().transpose(1, 2)
    t = torch.matmul(qs, ks.transpose(2, 3)).mul_(s["scale"])             # [sequence, K, g, own tokens]
    real_own = torch.arange(t.shape[-1], device=t.device) < s["suffix_len"][:, None]
    t.masked_fill_(~real_own[:, None, None, :], float("-inf"))
    # the largest value of a row over both parts, where the row is in either order
    at = torch.arange(n, device=q.device)
    group = torch.repeat_interleave(torch.arange(G, device=q.device), (off[1:] - off[:-1]).long(), output_size=n)
    slot = at - off[group]
    top_p = p.amax(-1).view(G, K, g, m)[group, :, :, slot]                # [sequence, K, g]
    top = torch.maximum(top_p, t.amax(-1))
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    t = torch.exp(t - top[..., None])
    total, acc = t.sum(-1), torch.matmul(t, vs)
    back = torch.zeros(G, m, K, g, device=q.device)
    back[group, slot] = top
    p.sub_(back.permute(0, 2, 3, 1).reshape(G, K, g * m, 1)).exp_()
    total = total + p.sum(-1).view(G, K, g, m)[group, :, :, slot]
    acc = acc + torch.matmul(p, v).view(G, K, g, m, D)[group, :, :, slot]
    total = torch.where(total == 0, torch.ones_like(total), total)
    s["out"].copy_((acc / total[..., None]).reshape(n, H, D))
    # what the rows received: own ones from their sequence, a prefix's from all that share it
    w = (t / total[..., None]).sum(2)                                     # [sequence, K, own tokens]
    s["suffix_weights"].copy_(torch.where(real_own[:, None], w, s["suffix_weights"]))
    inv = torch.zeros(G, m, K, g, device=q.device)
    inv[group, slot] = 1.0 / total
    w = p.mul_(inv.permute(0, 2, 3, 1).reshape(G, K, g * m, 1)).sum(2)    # [group, K, prefix tokens]
    s["prefix_weights"][:, rows[real]] = w.transpose(0, 1)[:, real]
    return s["out"], s["prefix_weights"], s["suffix_weights"]


def _plain_evict(s):
    packed, most, seg = s["packed"], s["most"], s["seg"]
    begin = seg[:-1] if packed else torch.zeros_like(seg)
    size = seg[1:] - seg[:-1] if packed else seg
    kept = size.clamp(max=s["n_keep"])
    n, t = size.numel(), torch.arange(most, device=seg.device)
    seqs = torch.arange(n, device=seg.device)
    real = t < size[:, None]
    rows = (begin[:, None] + t).clamp(max=s["weights"].shape[-1] - 1).long()
    w = s["weights"][:, rows].transpose(0, 1) if packed else s["weights"].gather(2, rows[:, None].expand(-1, s["weights"].shape[1], -1))
    stays = (t < s["first"]) | (t >= size[:, None] - s["recent"])
    w = torch.where(stays[:, None], torch.full_like(w, float("inf")), w).masked_fill_(~real[:, None], -1.0)      # [sequence, K, most]
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    chosen = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, (t < kept[:, None])[:, None].expand_as(w))
    b, h, row = chosen.nonzero(as_tuple=True)                             # ascending rows of every sequence and head
    if packed:
        s["seg_out"][1:] = torch.cumsum(kept, 0)
        to = torch.cumsum(chosen, -1)[b, h, row] - 1 + s["seg_out"][b]
        src, dst, where = (begin[b] + row, h), (to, h), (h, to)
        s["weights_out"][where] = s["weights"][h, begin[b] + row]
    else:
        s["seg_out"].copy_(kept)
        to = torch.cumsum(chosen, -1)[b, h, row] - 1
        src, dst, where = (b, row, h), (b, to, h), (b, h, to)
        s["weights_out"][where] = s["weights"][b, h, row]
    s["k_out"][dst] = s["k"][src]
    s["v_out"][dst] = s["v"][src]
    s["keep"][where] = row.to(torch.int32)
    return s["k_out"], s["v_out"], s["weights_out"], s["keep"], s["seg_out"]


def run(s):
    if own:
        return dict(rope=_own_rope, weights=_own_weights, step=_own_step, evict=_own_evict)[s["kind"]](s)
    return dict(rope=_plain_rope, weights=_plain_weights, step=_plain_step, evict=_plain_evict)[s["kind"]](s)


# ---- the definition in 64 bits -------------------------------------------------------------------------
def _exact_rope(c, s):
    """Pairs as complex numbers times exp(i angle); gradients by differentiation."""
    T, rot = s["q"].shape[0], c["rot"]
    axis = torch.tensor(_axes_of(c), device="cuda")
    angle = torch.stack([s["pos"][a].double() for a in axis.tolist()], 1) * s["inv_freq"].double()
    phase = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotated(x, gain):
        if c["norm"]:
            x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * gain
        r, rest = x[..., :rot], x[..., rot:]
        z = torch.complex(r[..., 0::2], r[..., 1::2]) if c["pairs"] else torch.complex(r[..., :rot // 2], r[..., rot // 2:])
        z = z * phase
        y = torch.stack([z.real, z.imag], -1).flatten(-2) if c["pairs"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([y, rest], -1)

    results, grads, gains = [], [], []
    for x, name in ((s["q"], "q"), (s["k"], "k")):
        x = x.double().requires_grad_(c["use"] == "train")
        gain = s["gain_" + name].double().requires_grad_(c["use"] == "train") if c["norm"] else None
        y = rotated(x, gain)
        results.append(y.detach())
        if c["use"] == "train":
            d = torch.autograd.grad(y, (x, gain) if c["norm"] else (x,), s[f"grad_{name}_out"].double())
            grads.append(d[0])
            gains += list(d[1:])
    if c["use"] == "train":
        return (*results, torch.cat(grads + [torch.zeros_like(grads[1])], 1), *gains)
    cache = s["cache"].double()
    for t, r in enumerate(s["row"].tolist()) if T <= 256 else [(slice(None), s["row"].long())]:
        cache[0][:, r] = results[1][t].transpose(0, 1) if T > 256 else results[1][t]
        cache[1][:, r] = s["v"][t].double().transpose(0, 1) if T > 256 else s["v"][t].double()
    return results[0], cache


def _exact_weights(c, s):
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    new, keys, count = _prompt_sizes(c)
    qo, ko = _offsets(new), _offsets(keys)
    out = torch.zeros(K, sum(keys), dtype=torch.float64, device="cuda")
    for b, (nq, nk, m) in enumerate(zip(new, keys, count)):
        for h in range(H):
            k = s["k"][ko[b]:ko[b + 1], h // (H // K)].double()
            for i in range(nq - m, nq, 4096):
                x = s["q"][qo[b] + i:qo[b] + min(i + 4096, nq), h].double() @ k.T / math.sqrt(D)
                if c["causal"]:
                    x.masked_fill_(torch.ones_like(x, dtype=torch.bool).triu(i + nk - nq + 1), -math.inf)
                out[h // (H // K), ko[b]:ko[b + 1]] += torch.softmax(x, -1).sum(0)
    return out


def _exact_step(c, s):
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    members, prefix, suffix = _step_sizes(c)
    starts, i = _offsets(prefix), 0
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    pw, sw = torch.zeros_like(s["prefix_weights"], dtype=torch.float64), torch.zeros_like(s["suffix_weights"], dtype=torch.float64)
    for group, n in enumerate(members):
        rows = slice(starts[group], starts[group + 1])
        pk, pv = s["prefix_k"][rows].double(), s["prefix_v"][rows].double()
        for _ in range(n):
            k = torch.cat([pk, s["suffix_k"][i, :suffix[i]].double()]).permute(1, 2, 0)
            v = torch.cat([pv, s["suffix_v"][i, :suffix[i]].double()]).permute(1, 0, 2)
            w = torch.softmax(s["q"][i].double().view(K, H // K, D) @ k / math.sqrt(D), dim=-1)
            out[i] = (w @ v).reshape(H, D)
            w = w.sum(1)
            pw[:, rows] += w[:, :prefix[group]]
            sw[i, :, :suffix[i]] = w[:, prefix[group]:]
            i += 1
    return out, pw, sw


def _exact_evict(c, s):
    """A sequence and a head at a time: rows sorted by (stays, weight, number)."""
    rows = _sizes(c["seqs"], c["rows"], c["ragged"], 5)
    at, to, n_out = _offsets(rows), 0, []
    res = [torch.zeros_like(s[x]) for x in ("k_out", "v_out", "weights_out", "keep")]
    for b, n in enumerate(rows):
        m = min(n, c["keep"])
        t = torch.arange(n)
        stays = (t < c["first"]) | (t >= n - c["recent"])
        for h in range(c["kv_heads"]):
            w = s["weights"][h, at[b]:at[b + 1]] if c["packed"] else s["weights"][b, h, :n]
            key = torch.where(stays, math.inf, w.cpu().double())
            kept = torch.argsort(-key, stable=True)[:m].sort().values.cuda()
            if c["packed"]:
                src, dst, where = (at[b] + kept, h), (slice(to, to + m), h), (h, slice(to, to + m))
            else:
                src, dst, where = (b, kept, h), (b, slice(0, m), h), (b, h, slice(0, m))
            res[0][dst], res[1][dst], res[2][where], res[3][where] = s["k"][src], s["v"][src], w[kept], kept.int()
        to += m
        n_out.append(to if c["packed"] else m)
    return (*(x.double() for x in res[:3]), res[3], _ints(([0] if c["packed"] else []) + n_out))


def exact(c, seed):
    return dict(rope=_exact_rope, weights=_exact_weights, step=_exact_step, evict=_exact_evict)[c["kind"]](c, prepare(c, seed))
