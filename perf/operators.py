"""The attention of a decoder layer as measurable cases: over whole prompts, its gradients, and for single
new tokens over a cache whose long beginning several sequences share.

The Skip-FFN block is the second half of a decoder layer; these operators are its first half.  Every token of
a packed batch attends (Section 4.2: skipped tokens stay in the attention), the keys and values of skipped
tokens leave the cache after the prefill (Section 4.3), and the tokens generated afterwards attend to what is
left.  Sizes: a LLaMA-3-8B layer (32 query heads, 8 key/value heads, 128 columns a head), LLaVA sequences of
576 visual + 40 text tokens, high-resolution sequences of 5 x 576 visual tokens, vision towers of 16 heads of 64
columns over 577 tokens, the repository's small layer (256 columns, 80 tokens), and generic ones.

  listed()   the fixed cases            draw(rng)  one more of the same ranges
  prepare()  what a program holds       run()      one pass over it
  work()     bytes and operations       exact()    the outputs in 64 bits
"""
from __future__ import annotations

import math
import random

import torch

own = False


# ---- the cases -------------------------------------------------------------------------------------
def prompt(name, *, seqs, tokens, past=0, ragged=0, heads=32, kv_heads=8, dim=128, causal=True, train=False):
    """`seqs` packed sequences of `tokens` new tokens each, after `past` tokens that the cache holds already.
    ragged != 0: sizes are drawn (from that number alone) between a fifth of those and the full size."""
    c = dict(kind="prompt", seqs=seqs, tokens=tokens, past=past, ragged=ragged, heads=heads, kv_heads=kv_heads,
             dim=dim, causal=causal, train=train)
    return dict(c, name=name) if name else c


def decode(name, *, seqs, shared, prefix, suffix, ragged=0, heads=32, kv_heads=8, dim=128):
    """One new token for each of `seqs` sequences.  `shared` sequences at a time have the same cached beginning of
    `prefix` tokens; each has up to `suffix` further tokens of its own."""
    c = dict(kind="decode", seqs=seqs, shared=shared, prefix=prefix, suffix=suffix, ragged=ragged, heads=heads,
             kv_heads=kv_heads, dim=dim)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the repository's small layer, one sequence of 64 visual + 16 text tokens: nothing but launches and latency
        prompt("prompt_small_layer", seqs=1, tokens=80, heads=4, kv_heads=4, dim=64),
        # a second question about four cached images: a few new tokens after a compacted cache
        prompt("append_b4", seqs=4, tokens=47, past=640, ragged=3),
        # the vision tower's attention, no mask: 8 images of 576 patches and a CLS token
        prompt("vision_b8", seqs=8, tokens=577, heads=16, kv_heads=16, dim=64, causal=False),
        # prefill of a batch of 8 requests
        prompt("prefill_b8", seqs=8, tokens=616),
        # prefill of 16 high-resolution requests of very different length
        prompt("prefill_ragged_b16", seqs=16, tokens=3080, ragged=4),
        # prefill of one long document
        prompt("prefill_long", seqs=1, tokens=16384),
        # a training step of the repository's small layer
        prompt("train_small_layer", seqs=1, tokens=80, heads=4, kv_heads=4, dim=64, train=True),
        # a training step of 16 sequences (the repository's default workload)
        prompt("train_b16", seqs=16, tokens=616, train=True),
        # a training step of 4 high-resolution sequences
        prompt("train_hd_b4", seqs=4, tokens=2944, train=True),
        # one decode step of 8 sequences, each with its own image of 144 retained + 40 text tokens
        decode("decode_b8", seqs=8, shared=1, prefix=184, suffix=64),
        # one decode step of 64 answers, 32 of them about each of two long inputs
        decode("decode_shared_b64", seqs=64, shared=32, prefix=5795, suffix=256, ragged=9),
        # one decode step of 4 sequences with long caches of their own
        decode("decode_long_b4", seqs=4, shared=1, prefix=32768, suffix=512, ragged=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 32), (16, 16), (16, 2), (12, 4), (28, 4), (8, 1), (6, 6)])
    dim = rng.choice([128, 128, 128, 64, 64, 80, 96, 40, 72])
    ragged = rng.choice([0, rng.randint(1, 10**6), rng.randint(1, 10**6)])
    kind = rng.choice(["prompt", "prompt", "append", "train", "train", "decode", "decode", "decode"])
    if kind == "decode":
        prefix, shared = _log(rng, 16, 32768), _log(rng, 1, 64)
        groups = max(1, min(_log(rng, 1, 32), 131072 // prefix))
        return decode(None, seqs=min(128, shared * groups), shared=shared, prefix=prefix, suffix=_log(rng, 1, 512), ragged=ragged,
                      heads=heads, kv_heads=kv_heads, dim=dim)
    if kind == "append":
        past = _log(rng, 100, 8192)
        return prompt(None, seqs=max(1, min(_log(rng, 1, 16), 16384 // past)), tokens=_log(rng, 1, 500), past=past, ragged=ragged,
                      heads=heads, kv_heads=kv_heads, dim=dim)
    tokens = _log(rng, 1, 8192 if kind == "prompt" else 4096)
    seqs = max(1, min(_log(rng, 1, 32), (32768 if kind == "prompt" else 12288) // tokens))
    return prompt(None, seqs=seqs, tokens=tokens, ragged=ragged, heads=heads, kv_heads=kv_heads, dim=dim,
                  causal=rng.random() < 0.8, train=kind == "train")


# ---- sizes that follow from a case -------------------------------------------------------------------
def _sizes(n, full, ragged, salt):
    if not ragged or not full:
        return [full] * n
    r = random.Random(ragged * 1000 + salt)
    return [r.randint(max(1, full // 5), full) for _ in range(n)]


def _prompt_sizes(c):
    """New tokens and visible keys of every sequence."""
    new, past = _sizes(c["seqs"], c["tokens"], c["ragged"], 1), _sizes(c["seqs"], c["past"], c["ragged"], 2)
    return new, [a + b for a, b in zip(new, past)]


def _decode_sizes(c):
    """Sequences of every group, its cached tokens, and every sequence's own tokens."""
    groups = -(-c["seqs"] // c["shared"])
    members = [min(c["shared"], c["seqs"] - i * c["shared"]) for i in range(groups)]
    return members, _sizes(groups, c["prefix"], c["ragged"], 3), _sizes(c["seqs"], c["suffix"], c["ragged"], 4)


def _offsets(sizes):
    out = [0]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def work(c):
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    if c["kind"] == "decode":
        members, prefix, suffix = _decode_sizes(c)
        seen = sum(m * p for m, p in zip(members, prefix)) + sum(suffix)
        return {"bytes": 2 * D * (2 * K * (sum(prefix) + sum(suffix)) + 2 * H * c["seqs"]), "flops": 4 * D * H * seen}
    new, keys = _prompt_sizes(c)
    pairs = sum(a * b - (a * (a - 1) // 2 if c["causal"] else 0) for a, b in zip(new, keys))
    once = 2 * D * (2 * H * sum(new) + 2 * K * sum(keys))      # q, out; k, v
    # a training step reads q, k, v and the output's gradient and writes the output and three gradients
    return {"bytes": 2 * once if c["train"] else once, "flops": (14 if c["train"] else 4) * D * H * pairs}


# ---- inputs --------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    s = dict(kind=c["kind"], scale=1.0 / math.sqrt(D))
    if c["kind"] == "decode":
        members, prefix, suffix = _decode_sizes(c)
        # a compacted cache keeps its capacity: [key/value head][token][column], of which the first rows are in use
        cap, own_cap = sum(prefix) + 64, c["suffix"] + 8
        cache, own_cache = _normal(gen, 2, K, cap, D), _normal(gen, 2, c["seqs"], K, own_cap, D)
        s.update(q=_normal(gen, c["seqs"], H, D), out=torch.empty(c["seqs"], H, D, dtype=torch.bfloat16, device="cuda"),
                 prefix_k=cache[0].transpose(0, 1), prefix_v=cache[1].transpose(0, 1),
                 suffix_k=own_cache[0].transpose(1, 2), suffix_v=own_cache[1].transpose(1, 2),
                 prefix_seg=_ints(_offsets(prefix)), group_off=_ints(_offsets(members)), suffix_len=_ints(suffix),
                 longest=max(prefix), members=max(members))
        return s
    new, keys = _prompt_sizes(c)
    T, Tk = sum(new), sum(keys)
    if c["past"]:
        # the cache of one layer holds the new tokens' keys and values too: [key/value head][token][column]
        cache = _normal(gen, 2, K, Tk, D)
        q, k, v = _normal(gen, T, H, D), cache[0].transpose(0, 1), cache[1].transpose(0, 1)
    else:
        # the projection's output, one row a token: query heads, key heads, value heads
        qkv = _normal(gen, T, H + 2 * K, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
    s.update(q=q, k=k, v=v, out=torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda"), causal=c["causal"], train=c["train"],
             seg_q=_ints(_offsets(new)), seg_k=_ints(_offsets(keys)), most_q=max(new), most_k=max(keys))
    if c["train"]:
        dqkv = torch.empty(T, H + 2 * K, D, dtype=torch.bfloat16, device="cuda")
        s.update(grad_out=_normal(gen, T, H, D), grad_q=dqkv[:, :H], grad_k=dqkv[:, H:H + K], grad_v=dqkv[:, H + K:])
    return s


# ---- one pass ------------------------------------------------------------------------------------------
def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _own_prompt(s):
    from paper_2503_21817_amd import binding as B
    (T, H, D), (Tk, K, _), n = s["q"].shape, s["k"].shape, s["seg_q"].numel() - 1
    if "workspace" not in s:
        s["workspace"] = _bytes(B.skipffn_attn_forward_workspace_bytes(T, Tk, n, H, K, D))
        if s["train"]:
            s["saved"] = _bytes(B.skipffn_attn_saved_bytes(T, H))
            s["backward_workspace"] = _bytes(B.skipffn_attn_backward_workspace_bytes(T, Tk, n, H, K, D))
    B.skipffn_attn_forward(s["q"], s["k"], s["v"], s["out"], s["seg_q"], s["seg_k"], causal=s["causal"], scale=s["scale"],
                           saved=s.get("saved"), workspace=s["workspace"])
    if not s["train"]:
        return s["out"]
    B.skipffn_attn_backward(s["q"], s["k"], s["v"], s["out"], s["grad_out"], s["seg_q"], s["seg_k"], s["saved"],
                            s["grad_q"], s["grad_k"], s["grad_v"], causal=s["causal"], scale=s["scale"],
                            workspace=s["backward_workspace"])
    return s["out"], s["grad_q"], s["grad_k"], s["grad_v"]


def _own_decode(s):
    from paper_2503_21817_amd import binding as B
    (n, H, D), (Tp, K, _) = s["q"].shape, s["prefix_k"].shape
    if "workspace" not in s:
        s["workspace"] = _bytes(B.skipffn_attn_decode_workspace_bytes(n, s["group_off"].numel() - 1, H, K, D, Tp, s["suffix_k"].shape[1]))
    B.skipffn_attn_decode(s["q"], s["prefix_k"], s["prefix_v"], s["prefix_seg"], s["group_off"], s["suffix_k"], s["suffix_v"],
                          s["suffix_len"], s["out"], scale=s["scale"], workspace=s["workspace"])
    return s["out"]


def _padded(x, seg, most):
    """Rows of packed sequences [T, heads, D] as [sequence, head, most, D] in float32 (rows past a sequence's end repeat one), and
    which of them are real."""
    at = torch.arange(most, device=x.device)
    real = at < (seg[1:] - seg[:-1])[:, None]
    rows = (seg[:-1, None] + at).clamp(max=x.shape[0] - 1).long()
    return x[rows].float().transpose(1, 2), real


def _packed(x, seg, T):
    """[sequence, head, most, D] back to [T, heads, D], rounded to bfloat16."""
    b = torch.repeat_interleave(torch.arange(seg.numel() - 1, device=x.device), (seg[1:] - seg[:-1]).long(), output_size=T)
    return x[b, :, torch.arange(T, device=x.device) - seg[b]].to(torch.bfloat16)


def _plain_prompt(s):
    (T, H, D), (Tk, K, _) = s["q"].shape, s["k"].shape
    seg_q, seg_k, n, g = s["seg_q"], s["seg_k"], s["seg_q"].numel() - 1, H // K
    q, real_q = _padded(s["q"], seg_q, s["most_q"])
    k, real_k = _padded(s["k"], seg_k, s["most_k"])
    v, _ = _padded(s["v"], seg_k, s["most_k"])
    mq, mk = s["most_q"], s["most_k"]
    q = q.reshape(n, K, g * mq, D)
    sees = real_q[:, :, None] & real_k[:, None, :]
    if s["causal"]:
        # a sequence's last query sees all its keys, the one before it all but one
        ahead = (seg_k[1:] - seg_k[:-1]) - (seg_q[1:] - seg_q[:-1])
        i, j = torch.arange(mq, device=q.device), torch.arange(mk, device=q.device)
        sees &= j[None, None, :] <= i[None, :, None] + ahead[:, None, None]
    p = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(n, K, g, mq, mk)
    p.masked_fill_(~sees[:, None, None], float("-inf"))
    top = p.amax(-1, keepdim=True)
    p.sub_(top.masked_fill_(top == float("-inf"), 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total.masked_fill_(total == 0, 1.0))
    p = p.view(n, K, g * mq, mk)
    o = torch.matmul(p, v)
    out = _packed(o.view(n, H, mq, D), seg_q, T)
    if not s["train"]:
        return out
    do, _ = _padded(s["grad_out"], seg_q, s["most_q"])
    do = do.reshape(n, K, g * mq, D)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    return out, _packed(dq.view(n, H, mq, D), seg_q, T), _packed(dk, seg_k, Tk), _packed(dv, seg_k, Tk)


def _plain_decode(s):
    (n, H, D), K = s["q"].shape, s["prefix_k"].shape[1]
    off, seg, m, g = s["group_off"], s["prefix_seg"], s["members"], H // K
    q, _ = _padded(s["q"], off, m)                                        # [group, H, member, D]
    G = q.shape[0]
    q = q.reshape(G, K, g * m, D)
    k, real = _padded(s["prefix_k"], seg, s["longest"])
    v, _ = _padded(s["prefix_v"], seg, s["longest"])
    p = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    p.masked_fill_(~real[:, None, None, :], float("-inf"))
    qs = s["q"].float().view(n, K, g, D)
    ks, vs = s["suffix_k"].float().transpose(1, 2), s["suffix_v"].float().transpose(1, 2)
    t = torch.matmul(qs, ks.transpose(2, 3)).mul_(s["scale"])             # [sequence, K, g, own tokens]
    t.masked_fill_((torch.arange(t.shape[-1], device=t.device) >= s["suffix_len"][:, None])[:, None, None, :], float("-inf"))
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
    return (acc / torch.where(total == 0, torch.ones_like(total), total)[..., None]).reshape(n, H, D).to(torch.bfloat16)


def run(s):
    if s["kind"] == "decode":
        return _own_decode(s) if own else _plain_decode(s)
    return _own_prompt(s) if own else _plain_prompt(s)


# ---- the definition in 64 bits -------------------------------------------------------------------------
def exact(c, seed):
    """softmax over a row's visible keys times the values, a sequence and a key/value head at a time; gradients by differentiation."""
    s = prepare(c, seed)
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    g, wide = H // K, torch.float64
    out = torch.zeros(s["q"].shape, dtype=wide, device="cuda")
    if c["kind"] == "decode":
        members, prefix, suffix = _decode_sizes(c)
        starts, i = _offsets(prefix), 0
        for group, count in enumerate(members):
            pk = s["prefix_k"][starts[group]:starts[group + 1]].to(wide)
            pv = s["prefix_v"][starts[group]:starts[group + 1]].to(wide)
            for _ in range(count):
                k = torch.cat([pk, s["suffix_k"][i, :suffix[i]].to(wide)]).permute(1, 2, 0)
                v = torch.cat([pv, s["suffix_v"][i, :suffix[i]].to(wide)]).permute(1, 0, 2)
                w = torch.softmax(s["q"][i].to(wide).view(K, g, D) @ k / math.sqrt(D), dim=-1)
                out[i] = (w @ v).reshape(H, D)
                i += 1
        return out
    new, keys = _prompt_sizes(c)
    qo, ko = _offsets(new), _offsets(keys)
    grads = [torch.zeros(s[x].shape, dtype=wide, device="cuda") for x in "qkv"] if c["train"] else None
    for b, (nq, nk) in enumerate(zip(new, keys)):
        hide = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1) if c["causal"] else None
        rq, rk = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        for h in range(K):
            q, k, v = (x.detach().to(wide).requires_grad_(c["train"])
                       for x in (s["q"][rq, h * g:(h + 1) * g], s["k"][rk, h], s["v"][rk, h]))
            rows = []
            for e in range(g):
                x = q[:, e] @ k.T / math.sqrt(D)
                rows.append(torch.softmax(x if hide is None else x.masked_fill(hide, -math.inf), dim=-1) @ v)
            o = torch.stack(rows, 1)
            out[rq, h * g:(h + 1) * g] = o.detach()
            if c["train"]:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["grad_out"][rq, h * g:(h + 1) * g].to(wide))
                grads[0][rq, h * g:(h + 1) * g], grads[1][rk, h], grads[2][rk, h] = dq, dk, dv
    return (out, *grads) if c["train"] else out
