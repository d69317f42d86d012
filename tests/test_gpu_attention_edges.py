"""Attention at the edges of what its tensors may be: inputs that repeat a row for every token, rows that lie over one another, one
token, scores without bounds."""
import numpy as np
import pytest
import torch

import test_gpu_attention as A
from test_gpu_attn_decode import Decode
from attn_bounds import assert_within, grad_bounds, out_bound
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of, to_dev_bf16

pytestmark = pytest.mark.gpu


def normal(rng, *shape):
    return to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal(shape)))


def step(q, k, v, g, nq, nk, causal, scale):
    """out, dq, dk, dv of a packed batch whose tensors end with its last row."""
    (T, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    seg_q, seg_k = A.offsets(nq), A.offsets(nk)
    out, dq = (torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dk, dv = (torch.full((Tk, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sizes = (T, Tk, len(nq), Hq, Hkv, D)
    saved = A.nbytes(B.skipffn_attn_saved_bytes(T, Hq))
    B.skipffn_attn_forward(q, k, v, out, seg_q, seg_k, causal=causal, scale=scale, saved=saved,
                           workspace=A.nbytes(B.skipffn_attn_forward_workspace_bytes(*sizes)))
    B.skipffn_attn_backward(q, k, v, out, g, seg_q, seg_k, saved, dq, dk, dv, causal=causal, scale=scale,
                            workspace=A.nbytes(B.skipffn_attn_backward_workspace_bytes(*sizes)))
    torch.cuda.synchronize()
    return out, dq, dk, dv


def check(q, k, v, g, got, nq, nk, causal, scale):
    q, k, v, g, out, dq, dk, dv = (f64_of(t.contiguous()) for t in (q, k, v, g, *got))
    aq = ak = 0
    for s, (n, m) in enumerate(zip(nq, nk)):
        rq, rk = slice(aq, aq + n), slice(ak, ak + m)
        aq, ak = aq + n, ak + m
        b = O.attn_backward_real(q[rq], k[rk], v[rk], g[rq], causal, scale)
        e = grad_bounds(q[rq], k[rk], v[rk], g[rq], scale, b)
        assert_within(out[rq], b["out"], out_bound(b["P"], v[rk], b["out"]), f"out, sequence {s}")
        for name, t, r in (("dq", dq, rq), ("dk", dk, rk), ("dv", dv, rk)):
            assert_within(t[r], b[name], e[name], f"{name}, sequence {s}")


# ---- rows past a sequence's end have no part in the gradients of its keys, whatever the strides make them read -----------------
@pytest.mark.parametrize("repeated", ["g", "q", "qg", "qkvg"])
@pytest.mark.parametrize("lens", [(50,), (33, 1, 95, 0, 64), (7, 130)], ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (2, 1, 128), (3, 3, 72)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_inputs_that_repeat_a_row_for_every_token(repeated, lens, Hq, Hkv, D, causal):
    """The gradient of a sum over tokens is one row expanded over them."""
    print(f"repeated {repeated} {lens} heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    rng, T = np.random.default_rng(D + len(lens)), sum(lens)
    t = [normal(rng, 1 if x in repeated else T, h, D).expand(T, h, D) for x, h in (("q", Hq), ("k", Hkv), ("v", Hkv), ("g", Hq))]
    got = step(*t, lens, lens, causal, 0.2)
    check(*t, got, lens, lens, causal, 0.2)
    same = step(*(x.contiguous() for x in t), lens, lens, causal, 0.2)
    assert all(np.array_equal(bits_of(a), bits_of(b)) for a, b in zip(got, same))


@pytest.mark.parametrize("stride", [8, 40, 64])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_rows_that_lie_over_one_another(stride, causal):
    """Token strides between 0 and the columns, heads apart."""
    H, D, lens = 2, 72, (50, 37, 3)
    print(f"rows {stride} apart, causal={causal}", flush=True)
    rng, T = np.random.default_rng(stride), sum(lens)
    t = []
    for _ in range(4):
        room = (T - 1) * stride + 128
        t.append(normal(rng, H * room).as_strided((T, H, D), (stride, room, 1)))
    got = step(*t, lens, lens, causal, 0.2)
    check(*t, got, lens, lens, causal, 0.2)
    same = step(*(x.contiguous() for x in t), lens, lens, causal, 0.2)
    assert all(np.array_equal(bits_of(a), bits_of(b)) for a, b in zip(got, same))


@pytest.mark.parametrize("nq,nk", [((1,), (1,)), ((1,), (40,)), ((1,), (3000,)), ((1, 0), (0, 5)), ((5,), (1,)), ((40,), (1,))], ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (5, 1, 128), (1, 1, 8)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_tensors_of_one_token(nq, nk, Hq, Hkv, D, causal):
    print(f"one token {nq} over {nk} heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    rng = np.random.default_rng(D + sum(nk))
    t = [normal(rng, n, h, D) for n, h in ((sum(nq), Hq), (sum(nk), Hkv), (sum(nk), Hkv), (sum(nq), Hq))]
    check(*t, step(*t, nq, nk, causal, 0.2), nq, nk, causal, 0.2)


@pytest.mark.parametrize("nq,nk", [((45, 20), (45, 20)), ((3, 40), (2500, 33)), ((70,), (31,))], ids=str)
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_one_row_for_every_token_and_head(nq, nk, causal):
    """Token and head strides of 0 in the queries and in the outputs' gradient, more keys or fewer than queries."""
    Hq, Hkv, D = 6, 2, 80
    print(f"one row {nq} over {nk} causal={causal}", flush=True)
    rng = np.random.default_rng(sum(nk))
    q, g = (normal(rng, 1, 1, D).expand(sum(nq), Hq, D) for _ in range(2))
    k, v = (normal(rng, sum(nk), Hkv, D) for _ in range(2))
    check(q, k, v, g, step(q, k, v, g, nq, nk, causal, 0.2), nq, nk, causal, 0.2)


def test_repeated_queries_of_large_scores():
    """Rows past the end that repeat a query have scores of some hundred and no log-sum-exp of their own."""
    lens, H, D = (41,), 2, 64
    rng = np.random.default_rng(1)
    q = (20.0 * normal(rng, 1, H, D)).expand(41, H, D)
    k, v, g = (normal(rng, 41, H, D) for _ in range(3))
    got = step(q, k, v, g, lens, lens, True, 1.0)
    same = step(q.contiguous(), k, v, g, lens, lens, True, 1.0)
    assert all(np.array_equal(bits_of(a), bits_of(b)) for a, b in zip(got, same))
    assert all(torch.isfinite(t.float()).all() for t in got)


# ---- a row's bits are its own: neither a neighbour's queries nor keys that it does not see change its rounding --------------------
@pytest.mark.parametrize("Hq,Hkv,D,nq,nk", [(4, 2, 128, (200, 70), (200, 70)), (4, 4, 64, (200, 130), (200, 130)), (32, 8, 128, (150,) * 9, (150,) * 9),
                                            (8, 2, 80, (40,), (3000,))], ids=str)
def test_a_query_or_an_unseen_key_leaves_the_other_rows_bits(Hq, Hkv, D, nq, nk):
    print(f"neighbours, heads {Hq}/{Hkv} D={D} {nq} over {nk}", flush=True)
    p = A.Prompt(nq, nk, Hq, Hkv, D, "fused" if nq == nk else "plain")
    p.q[..., 0] = 1.0
    p.forward(True, 0.2)
    torch.cuda.synchronize()
    clean, stat = bits_of(p.out), p.saved[:4 * p.T * Hq].view(torch.float32).view(Hq, p.T).clone()
    q, k = p.q.clone(), p.k.clone()
    hit = np.zeros(clean.shape[:2], bool)
    row = nq[0] - 20                                     # a query of large scores among ordinary ones
    p.q[row] *= 64.0
    hit[row] = True
    key = nk[0] - 15                                     # a key of infinite scores, seen by the last rows of the first sequence
    p.k[key, 0, 0] = float("inf")
    hit[nq[0] - 15:nq[0], :Hq // Hkv] = True
    p.forward(True, 0.2)
    torch.cuda.synchronize()
    after = p.saved[:4 * p.T * Hq].view(torch.float32).view(Hq, p.T)
    rows = ~hit[:sum(nq)]
    assert np.array_equal(bits_of(p.out)[:sum(nq)][rows], clean[:sum(nq)][rows])
    assert torch.equal(after[:, :sum(nq)].T[torch.from_numpy(rows).cuda()], stat[:, :sum(nq)].T[torch.from_numpy(rows).cuda()])
    assert np.isnan(f64_of(p.out)[nq[0] - 15:nq[0], :Hq // Hkv]).all()
    p.q.copy_(q)
    p.k.copy_(k)
    p.forward(True, 0.2)
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(p.out), clean)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 1, 64)])
def test_a_sequence_leaves_the_bits_of_those_that_share_its_prefix(Hq, Hkv, D):
    d = Decode((6, 0), (900,), (40, 33, 0, 70, 5, 1), Hq, Hkv, D)
    d.q[..., 0] = 1.0
    d.run(0.2)
    torch.cuda.synchronize()
    clean = bits_of(d.out)
    d.q[2] *= 64.0
    d.sk[3, 60, :, 0] = float("inf")
    d.run(0.2)
    torch.cuda.synchronize()
    got = bits_of(d.out)
    assert np.array_equal(got[[0, 1, 4, 5]], clean[[0, 1, 4, 5]])
    assert np.isnan(f64_of(d.out)[3]).all() and np.isfinite(f64_of(d.out)[2]).all()


# ---- a row that sees keys, all with scores of minus infinity: 0 / 0, not the zeros of a row that sees none ------------------------
def against_all_but(keys, q, k):
    """Every query's product with the keys listed is minus infinity."""
    q[..., 0] = -1.0
    k[keys, :, 0] = float("inf")


@pytest.mark.parametrize("Hq,Hkv,D,lens", [(4, 2, 128, (70, 45)), (4, 4, 64, (33, 130)), (32, 8, 128, (150,) * 9), (6, 2, 96, (40, 40))], ids=str)
def test_a_row_whose_every_score_is_minus_infinity(Hq, Hkv, D, lens):
    print(f"minus infinity, heads {Hq}/{Hkv} D={D} {lens}", flush=True)
    p = A.Prompt(lens, lens, Hq, Hkv, D)
    p.forward(True, 0.2)
    p.backward(True, 0.2)
    torch.cuda.synchronize()
    clean = [bits_of(t) for t in (p.out, p.dq, p.dk, p.dv)]
    n = lens[0]
    against_all_but([0], p.q[:n], p.k[:n])               # the first row sees the first key alone
    p.forward(True, 0.2)
    p.backward(True, 0.2)
    torch.cuda.synchronize()
    out = f64_of(p.out)
    assert np.isnan(out[0]).all() and np.isnan(f64_of(p.dq)[0]).all() and np.isnan(f64_of(p.dv)[0]).all()
    # the others as if the key were not there
    q, k, v = (f64_of(t)[1:n] for t in (p.q, p.k, p.v))
    want, P = O.attn_forward_real(q, k, v, True, 0.2)
    assert_within(out[1:n], want, out_bound(P, v, want), "out")
    for t, c in zip((p.out, p.dq, p.dk, p.dv), clean):   # and nothing of it in the next sequences
        assert np.array_equal(bits_of(t)[n:], c[n:])
    against_all_but(slice(0, n), p.q[:n], p.k[:n])
    for causal in (True, False):
        p.forward(causal, 0.2)
        torch.cuda.synchronize()
        assert np.isnan(f64_of(p.out)[:n]).all() and np.isfinite(f64_of(p.out)[n:sum(lens)]).all()


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_parts_whose_every_score_is_minus_infinity(Hq, Hkv, D, causal):
    """Keys cut into parts: some parts of nothing but such scores have weight 0; if all are, the row is not a number."""
    nq, nk = (9, 20), (5, 4500)
    print(f"minus infinity in parts, heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    for hidden in (slice(0, 3000), slice(1000, 4400), slice(0, 4500)):
        p = A.Prompt(nq, nk, Hq, Hkv, D, "cache")
        assert p.fws.numel() > 16
        q, k, v = p.q[9:29], p.k[5:4505], p.v[5:4505]
        against_all_but(hidden, q, k)
        p.forward(causal, 0.2)
        torch.cuda.synchronize()
        out = f64_of(p.out)
        if causal:
            assert np.all(out[:4] == 0)                  # these see no key
        assert np.isfinite(out[:9]).all()
        if hidden == slice(0, 4500):
            assert np.isnan(out[9:29]).all()
            continue
        keep = np.ones(4500, bool)
        keep[hidden] = False
        f = [f64_of(t) for t in (q, k, v)]
        want, weights = np.zeros(f[0].shape), np.zeros((Hq, 20, 4500))
        for i in range(20):                              # row i sees the first nk - nq + 1 + i keys
            sees = keep & (np.arange(4500) <= 4480 + i if causal else True)
            want[i:i + 1], P = O.attn_forward_real(f[0][i:i + 1], f[1][sees], f[2][sees], False, 0.2)
            weights[:, i, sees] = P[:, 0]
        assert_within(out[9:29], want, out_bound(weights, f[2], want), f"out without {hidden}")


@pytest.mark.parametrize("prefix", [0, 70, 3000])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 1, 64)])
def test_single_tokens_whose_every_score_is_minus_infinity(prefix, Hq, Hkv, D):
    print(f"minus infinity, single tokens, prefix {prefix}, heads {Hq}/{Hkv} D={D}", flush=True)
    d = Decode((4, 0), (prefix,), (40, 0, 300, 7), Hq, Hkv, D)
    d.q[..., 0] = -1.0
    d.sk[0, :, :, 0] = float("inf")
    d.sk[2, 30:, :, 0] = float("inf")
    d.run(0.2)
    torch.cuda.synchronize()
    out = f64_of(d.out)
    if prefix == 0:
        assert np.isnan(out[0]).all() and np.all(out[1] == 0)
    f = {n: f64_of(getattr(d, n)) for n in ("q", "pk", "pv", "sk", "sv")}
    want, seen = O.attn_decode_real(f["q"], f["pk"], f["pv"], d.seg, d.off, f["sk"], f["sv"], [0, 0, 30, 7], 0.2)
    for i, (k, v, P) in enumerate(seen):                 # the rows of such scores as if they were not there
        if i > 0 or prefix > 0:
            assert_within(out[i:i + 1], want[i:i + 1], out_bound(P[:, None], v, want[i:i + 1]), f"sequence {i}")
    d.pk[..., 0] = float("inf")
    d.run(0.2)
    torch.cuda.synchronize()
    out = f64_of(d.out)
    assert np.isnan(out[0]).all() and np.isfinite(out[2:]).all()
    assert np.isnan(out[1]).all() if prefix > 0 else np.all(out[1] == 0)


# ---- gradients of peaked rows ------------------------------------------------------------------------------------------------
def test_gradients_of_peaked_rows():
    """Queries of 30 times the usual size, as in the forward's test: weights are formed again from scores and log-sum-exps of some hundred,
    and those of keys that a row does not see overflow before they are masked."""
    lens, H, D, scale = (257, 90, 33), 2, 64, 0.125
    p = A.Prompt(lens, lens, H, H, D, "plain", q_std=30.0)
    p.forward(True, scale)
    p.backward(True, scale)
    torch.cuda.synchronize()
    f, a = {n: f64_of(getattr(p, n)) for n in ("q", "k", "v", "g", "dq", "dk", "dv")}, 0
    for s, n in enumerate(lens):
        r = slice(a, a + n)
        a += n
        q, k, v, g = (f[x][r] for x in "qkvg")
        b = O.attn_backward_real(q, k, v, g, True, scale)
        e = grad_bounds(q, k, v, g, scale, b)
        # a score, and the log-sum-exp, is off by up to 0.0014 in the exponent: a weight by eta of itself.  out is then off by eta A with A = P |v|
        # more, so delta by |g| . eta A, dS by eta |dS| + P (that), and what is summed from them accordingly
        eta = 0.002
        for h in range(H):
            A_ = b["P"][h] @ np.abs(v[:, h])
            E = eta * (np.abs(b["dS"][h]) + b["P"][h] * (np.abs(g[:, h]) * A_).sum(axis=1, keepdims=True))
            e["dq"][:, h] += 1.1 * scale * (E @ np.abs(k[:, h]))
            e["dk"][:, h] += 1.1 * scale * (E.T @ np.abs(q[:, h]))
            e["dv"][:, h] += 1.1 * eta * (b["P"][h].T @ np.abs(g[:, h]))
        for name in ("dq", "dk", "dv"):
            assert_within(f[name][r], b[name], e[name], f"{name}, sequence {s}")
