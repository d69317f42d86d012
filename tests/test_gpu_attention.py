"""Attention over packed prompts and its gradients through the C ABI against the oracle, element by element within the
bounds of attn_bounds."""
import numpy as np
import pytest
import torch

from attn_bounds import assert_within, grad_bounds, out_bound
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of, to_dev_bf16

pytestmark = pytest.mark.gpu

BEHIND = 3           # rows behind the last sequence


def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()


def nbytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


class Prompt:
    """Inputs on the device in one of the layouts a program has them in: `fused` (column ranges of one projection's output),
    `cache` (k, v by head), `plain` (a tensor each).  Behind the last sequence there are rows of NaN."""

    def __init__(self, nq, nk, Hq, Hkv, D, layout="fused", seed=0, q_std=1.0):
        rng = np.random.default_rng(seed + sum(nq) + D)
        self.nq, self.nk, self.Hq, self.Hkv, self.D = list(nq), list(nk), Hq, Hkv, D
        self.T, self.Tk = sum(nq) + BEHIND, sum(nk) + BEHIND
        if layout == "fused":
            assert nq == nk
            self.all = self._bits(rng, self.T, Hq + 2 * Hkv)
            t = to_dev_bf16(self.all)
            self.q, self.k, self.v = t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]
            g = torch.full((self.T, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
            self.dq, self.dk, self.dv = g[:, :Hq], g[:, Hq:Hq + Hkv], g[:, Hq + Hkv:]
        else:
            self.q = to_dev_bf16(self._bits(rng, self.T, Hq, q_std))
            kv = [to_dev_bf16(self._bits(rng, self.Tk, Hkv)) for _ in range(2)]
            if layout == "cache":
                kv = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in kv]
            self.k, self.v = kv
            self.dq, self.dk, self.dv = (torch.full_like(t, 7.0) for t in (self.q, self.k, self.v))
        self.g = to_dev_bf16(self._bits(rng, self.T, Hq))
        self.out = torch.full((self.T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.seg_q, self.seg_k = offsets(nq), None if nq == nk else offsets(nk)
        self.saved = nbytes(B.skipffn_attn_saved_bytes(self.T, Hq))
        sizes = (self.T, self.Tk, len(nq), Hq, Hkv, D)
        self.fws, self.bws = nbytes(B.skipffn_attn_forward_workspace_bytes(*sizes)), nbytes(B.skipffn_attn_backward_workspace_bytes(*sizes))

    def _bits(self, rng, T, H, std=1.0):
        x = rng.standard_normal((T, H, self.D)) * std
        x[T - BEHIND:] = np.nan
        return O.f64_to_bf16_bits(x)

    def forward(self, causal, scale, saved=True):
        B.skipffn_attn_forward(self.q, self.k, self.v, self.out, self.seg_q, self.seg_k, causal=causal, scale=scale,
                               saved=self.saved if saved else None, workspace=self.fws)

    def backward(self, causal, scale):
        B.skipffn_attn_backward(self.q, self.k, self.v, self.out, self.g, self.seg_q, self.seg_k, self.saved, self.dq, self.dk,
                                self.dv, causal=causal, scale=scale, workspace=self.bws)

    def check(self, causal, scale, gradients):
        torch.cuda.synchronize()
        f = {n: f64_of(getattr(self, n)) for n in ("q", "k", "v", "g", "out", "dq", "dk", "dv")}
        aq = ak = 0
        for s, (nq, nk) in enumerate(zip(self.nq, self.nk)):
            rq, rk = slice(aq, aq + nq), slice(ak, ak + nk)
            aq, ak = aq + nq, ak + nk
            q, k, v, g = f["q"][rq], f["k"][rk], f["v"][rk], f["g"][rq]
            b = O.attn_backward_real(q, k, v, g, causal, scale)
            assert_within(f["out"][rq], b["out"], out_bound(b["P"], v, b["out"]), f"out, sequence {s}")
            if gradients:
                e = grad_bounds(q, k, v, g, scale, b)
                for n, r in (("dq", rq), ("dk", rk), ("dv", rk)):
                    assert_within(f[n][r], b[n], e[n], f"{n}, sequence {s}")
        assert np.all(f["out"][aq:] == 7.0)
        assert np.all(f["dq"][aq if gradients else 0:] == 7.0)
        assert all(np.all(f[n][ak if gradients else 0:] == 7.0) for n in ("dk", "dv"))


LENGTHS = [(1,), (31, 0, 33, 64), (129, 65, 1, 128), (300, 17), (63, 32, 2)]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 128), (3, 3, 64), (6, 2, 80), (5, 1, 40), (8, 2, 96), (2, 2, 8)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_packed_sequences_forward_and_backward(lens, Hq, Hkv, D, causal):
    print(f"attention {lens} heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    p = Prompt(lens, lens, Hq, Hkv, D, "fused")
    p.forward(causal, D ** -0.5)
    p.backward(causal, D ** -0.5)
    p.check(causal, D ** -0.5, True)


@pytest.mark.parametrize("nq,nk", [((1, 1, 1), (1, 300, 64)), ((40, 7), (333, 7)), ((50, 64, 3), (20, 63, 0)), ((5, 0, 9), (0, 70, 129)),
                                   ((130,), (1000,))], ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (2, 2, 64), (6, 2, 72)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("layout", ["cache", "plain"])
def test_queries_after_or_beyond_their_keys(nq, nk, Hq, Hkv, D, causal, layout):
    """More keys than queries (new tokens after cached ones), fewer (rows that see nothing), none."""
    print(f"attention {nq} over {nk} heads {Hq}/{Hkv} D={D} causal={causal} {layout}", flush=True)
    p = Prompt(nq, nk, Hq, Hkv, D, layout)
    p.forward(causal, 0.11)
    p.backward(causal, 0.11)
    p.check(causal, 0.11, True)


def test_inference_writes_no_statistics_and_the_same_rows():
    p = Prompt((70, 200), (70, 200), 4, 2, 128)
    p.forward(True, 0.1)
    want = bits_of(p.out)
    p.out.fill_(7.0)
    p.saved.fill_(0xA5)
    p.forward(True, 0.1, saved=False)
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(p.out), want) and bool((p.saved == 0xA5).all())


def test_peaked_softmax_and_large_scores():
    """Queries of 30 times the usual size: weights of nearly 0 and 1, scores of some hundred, maxima that grow along the row."""
    p = Prompt((257, 90), (257, 90), 2, 2, 64, "plain", q_std=30.0)
    f = {n: f64_of(getattr(p, n)) for n in "qkv"}
    p.forward(True, 0.125)
    torch.cuda.synchronize()
    got, a = f64_of(p.out), 0
    for n in p.nq:
        r = slice(a, a + n)
        a += n
        out, P = O.attn_forward_real(f["q"][r], f["k"][r], f["v"][r], True, 0.125)
        # a score is off by up to 64 products of 2^-24 |q| |k| scale log2(e): |q| . |k| is about 64 x 30 x 0.64, so 0.0014 in the exponent
        extra = 0.001 * 2 * np.stack([P[h] @ np.abs(f["v"][r][:, h]) for h in range(2)], axis=1)
        assert_within(got[r], out, out_bound(P, f["v"][r], out) + extra, "out")


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (2, 1, 128)])
def test_more_sequences_than_lanes(Hq, Hkv, D):
    rng = np.random.default_rng(D)
    lens = tuple(int(n) for n in rng.integers(0, 70, 150))
    print(f"attention {len(lens)} sequences heads {Hq}/{Hkv} D={D}", flush=True)
    p = Prompt(lens, lens, Hq, Hkv, D)
    p.forward(True, D ** -0.5)
    p.backward(True, D ** -0.5)
    p.check(True, D ** -0.5, True)


@pytest.mark.parametrize("lens,Hq,Hkv,D,causal", [((257, 130, 64, 1, 190, 33, 250, 97) * 4, 32, 8, 128, True),
                                                  ((200,) * 24, 24, 24, 64, False), ((150, 31, 260) * 9, 12, 4, 96, True)])
def test_more_pieces_than_fit_the_chip(lens, Hq, Hkv, D, causal):
    """Workgroups go on to further pieces, of other sequences, heads and lengths; twice the same bits."""
    print(f"attention {len(lens)} sequences heads {Hq}/{Hkv} D={D}", flush=True)
    p = Prompt(lens, lens, Hq, Hkv, D)
    p.forward(causal, D ** -0.5)
    p.backward(causal, D ** -0.5)
    p.check(causal, D ** -0.5, True)
    first = [bits_of(t) for t in (p.out, p.dq, p.dk, p.dv)]
    for t in (p.out, p.dq, p.dk, p.dv):
        t.fill_(7.0)
    p.forward(causal, D ** -0.5)
    p.backward(causal, D ** -0.5)
    torch.cuda.synchronize()
    assert all(np.array_equal(bits_of(t), f) for t, f in zip((p.out, p.dq, p.dk, p.dv), first))


@pytest.mark.parametrize("nq,nk", [((3,), (4000,)), ((40, 1, 0, 17), (3000, 2100, 0, 5000)), ((9, 20), (5, 2500))], ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 4, 64), (6, 1, 80)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_few_queries_whose_keys_are_cut_into_parts(nq, nk, Hq, Hkv, D, causal):
    print(f"attention {nq} over {nk} heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    p = Prompt(nq, nk, Hq, Hkv, D, "cache")
    assert p.fws.numel() > 16                             # the forward call wants room for parts
    p.forward(causal, D ** -0.5)
    p.backward(causal, D ** -0.5)
    p.check(causal, D ** -0.5, True)


def test_inputs_that_repeat_and_odd_strides():
    """Keys and values of stride 0 by head (one head seen as several) and by token, rows with a gap between them: the same bits as
    from tensors that hold the repeats."""
    T, H, D = 75, 4, 64
    rng = np.random.default_rng(9)
    seg = offsets((50, 25))
    wide = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((T, H + 3, D + 8))))
    q, g = wide[:, 1:H + 1, :D], wide[:, 2:H + 2, :D]
    one = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((2, T, 1, D))))
    row = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((1, H, D))))
    for k, v in ((one[0].expand(T, H, D), one[1].expand(T, H, D)), (row.expand(T, H, D), one[1].expand(T, H, D))):
        got = []
        for a, b, c, d in ((q, k, v, g), tuple(t.contiguous() for t in (q, k, v, g))):
            out, dq, dk, dv = (torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(4))
            saved, ws = nbytes(B.skipffn_attn_saved_bytes(T, H)), nbytes(B.skipffn_attn_backward_workspace_bytes(T, T, 2, H, H, D))
            B.skipffn_attn_forward(a, b, c, out, seg, saved=saved)
            B.skipffn_attn_backward(a, b, c, out, d, seg, None, saved, dq, dk, dv, workspace=ws)
            got.append([bits_of(t) for t in (out, dq, dk, dv)])
        assert all(np.array_equal(x, y) for x, y in zip(*got))


def test_a_sequence_that_is_not_finite_leaves_the_others_as_they_are():
    """NaN and infinities in one sequence reach nothing of its neighbours, in either direction and pass."""
    lens, Hq, Hkv, D = (45, 70, 33), 4, 2, 128
    p = Prompt(lens, lens, Hq, Hkv, D)
    p.forward(True, 0.1)
    p.backward(True, 0.1)
    torch.cuda.synchronize()
    clean = [bits_of(t) for t in (p.out, p.dq, p.dk, p.dv)]
    p.v[45:115] = float("nan")
    p.k[60] = float("inf")
    p.q[70, 1] = float("-inf")
    p.g[80] = float("nan")
    p.forward(True, 0.1)
    p.backward(True, 0.1)
    torch.cuda.synchronize()
    for t, c in zip((p.out, p.dq, p.dk, p.dv), clean):
        b = bits_of(t)
        assert np.array_equal(b[:45], c[:45]) and np.array_equal(b[115:], c[115:])
    assert np.all(np.isnan(f64_of(p.out)[45:115]))


def test_keys_past_32_bits():
    """Queries after a cache whose rows lie past 2^31 elements."""
    Hq, Hkv, D, Tk, n = 4, 8, 128, 2_200_000, 200
    rng = np.random.default_rng(4)
    Hq = 8
    bits = O.f64_to_bf16_bits(rng.standard_normal((2, n, Hkv, D)))
    kv = [torch.zeros(Tk, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for t, b in zip(kv, bits):
        t[Tk - n:] = to_dev_bf16(b)
    q = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((50, Hq, D))))
    out = torch.empty_like(q)
    seg_q, seg_k = offsets((50,)), torch.tensor([Tk - n, Tk], dtype=torch.int32, device="cuda")
    B.skipffn_attn_forward(q, *kv, out, seg_q, seg_k, workspace=nbytes(B.skipffn_attn_forward_workspace_bytes(50, Tk, 1, Hq, Hkv, D)))
    torch.cuda.synchronize()
    f = O.bf16_bits_to_f64(bits)
    want, P = O.attn_forward_real(f64_of(q), f[0], f[1], True, D ** -0.5)
    assert_within(f64_of(out), want, out_bound(P, f[1], want), "out")


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_gradients_against_differences(causal):
    """Along random directions of q, k and v the outputs' change, in fp64 by the oracle, is what the gradients say."""
    Hq, Hkv, D, lens = 4, 2, 64, (37, 64)
    p = Prompt(lens, lens, Hq, Hkv, D, "plain")
    p.forward(causal, 0.125)
    p.backward(causal, 0.125)
    torch.cuda.synchronize()
    f = {n: f64_of(getattr(p, n)) for n in ("q", "k", "v", "g", "dq", "dk", "dv")}
    rng, eps, a = np.random.default_rng(5), 1e-5, 0
    for n in lens:
        r = slice(a, a + n)
        a += n
        x = {m: f[m][r] for m in ("q", "k", "v")}
        b = O.attn_backward_real(x["q"], x["k"], x["v"], f["g"][r], causal, 0.125)
        e = grad_bounds(x["q"], x["k"], x["v"], f["g"][r], 0.125, b)
        for m in x:
            d = rng.standard_normal(x[m].shape)
            def loss(t):
                y = dict(x, **{m: x[m] + t * d})
                return (O.attn_forward_real(y["q"], y["k"], y["v"], causal, 0.125)[0] * f["g"][r]).sum()
            by_difference = (loss(eps) - loss(-eps)) / (2 * eps)
            # every element's bound in the worst direction, and the differences' own error (eps^2, 1e-16 / eps)
            allowed = (e["d" + m] * np.abs(d)).sum() + 1e-4 * np.abs(by_difference) + 1e-4
            assert abs((f["d" + m][r] * d).sum() - by_difference) <= allowed


@pytest.mark.parametrize("Hq,Hkv,D,nq,nk", [(4, 2, 128, (200, 40), (200, 40)), (32, 8, 128, (150,) * 9, (150,) * 9), (4, 4, 64, (130,), (130,)),
                                            (8, 2, 80, (5, 60), (3000, 60)), (6, 3, 96, (150,) * 20, (150,) * 20)], ids=str)
def test_values_that_are_not_finite_reach_the_rows_that_see_them_alone(Hq, Hkv, D, nq, nk):
    """In a causal prompt a NaN or an infinity among the values of token j shows in the rows from j on, in its column; the rows before it
    keep their bits, and so do the other columns."""
    print(f"not finite, heads {Hq}/{Hkv} D={D} {nq} over {nk}", flush=True)
    p = Prompt(nq, nk, Hq, Hkv, D, "fused" if nq == nk else "plain")
    p.forward(True, D ** -0.5)
    torch.cuda.synchronize()
    clean, lse = bits_of(p.out), p.saved.clone()
    ko, qo = np.concatenate([[0], np.cumsum(nk)]), np.concatenate([[0], np.cumsum(nq)])
    planted = []                                         # (sequence, key, key/value head, column, value)
    for s, (a, b) in enumerate(zip(nq, nk)):
        for back, value in ((a // 2, np.inf), (1, np.nan), (a - 1, -np.inf)):
            key, kh, col = b - 1 - back, s % Hkv, (7 * s + 3 * back) % D
            planted.append((s, key, kh, col, value))
            p.v[int(ko[s]) + key, kh, col] = value
    p.forward(True, D ** -0.5)
    torch.cuda.synchronize()
    got, f = bits_of(p.out), f64_of(p.out)
    hit = np.zeros(got.shape, bool)
    for s, key, kh, col, value in planted:
        first = max(key - (nk[s] - nq[s]), 0)            # the first query that sees the key
        heads = slice(kh * (Hq // Hkv), (kh + 1) * (Hq // Hkv))
        hit[qo[s] + first:qo[s + 1], heads, col] = True
    assert np.array_equal(got[~hit], clean[~hit])
    assert not np.isfinite(f[hit]).any()
    assert torch.equal(p.saved[:4 * p.T * Hq], lse[:4 * p.T * Hq])


def torch_check(p, causal, scale, heads, gradients):
    """The same bounds as Prompt.check, in fp64 on the device, of the key/value heads listed."""
    from attn_bounds import F, P16, SLACK, U
    rep = p.Hq // p.Hkv
    aq = ak = 0
    for s, (nq, nk) in enumerate(zip(p.nq, p.nk)):
        rq, rk = slice(aq, aq + nq), slice(ak, ak + nk)
        aq, ak = aq + nq, ak + nk
        hide = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1) if causal else None
        for kh in heads:
            k, v = p.k[rk, kh].double(), p.v[rk, kh].double()
            dk, dv, ek, ev = (torch.zeros_like(k) for _ in range(4))
            for h in range(kh * rep, (kh + 1) * rep):
                q, g = p.q[rq, h].double(), p.g[rq, h].double()
                S = scale * (q @ k.T)
                P = torch.softmax(S if hide is None else S.masked_fill(hide, -float("inf")), -1)
                del S
                out = P @ v
                e_out = SLACK * ((U + F) * (P @ v.abs()) + U * out.abs())
                assert bool(((p.out[rq, h].double() - out).abs() <= e_out).all()), ("out", s, h)
                if not gradients:
                    continue
                e_delta = (g.abs() * (e_out + P16 * out.abs())).sum(1, keepdim=True)
                dS = P * (g @ v.T - (g * out).sum(1, keepdim=True))
                E = P * (e_delta + P16 * (g.abs() @ v.abs().T)) + (U + F) * dS.abs()
                dq = scale * (dS @ k)
                bound = SLACK * (scale * (E @ k.abs()) + U * dq.abs())
                assert bool(((p.dq[rq, h].double() - dq).abs() <= bound).all()), ("dq", s, h)
                dk += scale * (dS.T @ q)
                dv += P.T @ g
                ek += scale * (E.T @ q.abs())
                ev += (U + F) * (P.T @ g.abs())
            if gradients:
                assert bool(((p.dk[rk, kh].double() - dk).abs() <= SLACK * (ek + U * dk.abs())).all()), ("dk", s, kh)
                assert bool(((p.dv[rk, kh].double() - dv).abs() <= SLACK * (ev + U * dv.abs())).all()), ("dv", s, kh)


@pytest.mark.parametrize("lens,Hq,Hkv,D,causal,heads", [((2944, 616, 1), 32, 8, 128, True, (0, 7)), ((577,) * 4, 16, 16, 64, False, (3, 15)),
                                                        ((3500, 40), 28, 4, 96, True, (2,))], ids=str)
def test_full_size_forward_and_backward(lens, Hq, Hkv, D, causal, heads):
    print(f"attention {lens} heads {Hq}/{Hkv} D={D} causal={causal}", flush=True)
    p = Prompt(lens, lens, Hq, Hkv, D)
    p.forward(causal, D ** -0.5)
    p.backward(causal, D ** -0.5)
    torch.cuda.synchronize()
    torch_check(p, causal, D ** -0.5, heads, True)


def test_full_size_long_prompt():
    p = Prompt((16384,), (16384,), 8, 2, 128)
    p.forward(True, 128 ** -0.5)
    torch.cuda.synchronize()
    torch_check(p, True, 128 ** -0.5, (0, 1), False)


@pytest.mark.parametrize("Hq,Hkv,D", [(40, 1, 64), (33, 1, 128), (64, 2, 24)])
def test_many_query_heads_a_key_value_head(Hq, Hkv, D):
    lens = (65, 33, 4)
    p = Prompt(lens, lens, Hq, Hkv, D)
    p.forward(True, D ** -0.5)
    p.backward(True, D ** -0.5)
    p.check(True, D ** -0.5, True)


def test_results_in_column_ranges_and_by_head():
    """out and the gradients as column ranges of wider rows, and as [head][token][column]: the same bits, and nothing between them."""
    T, Hq, Hkv, D, lens = 133, 4, 2, 72, (100, 30)
    p = Prompt(lens, lens, Hq, Hkv, D, "plain")
    p.forward(True, 0.1)
    p.backward(True, 0.1)
    torch.cuda.synchronize()
    want = [bits_of(t) for t in (p.out, p.dq, p.dk, p.dv)]
    wide = torch.full((T, 20, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    other = torch.full((T, 6, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    ranges = [other[:, 1:1 + Hq, 8:], wide[:, 6:6 + Hq, 8:], wide[:, 11:11 + Hkv, 8:], wide[:, 15:15 + Hkv, 8:]]
    byhead = [torch.full((h, T + 3, D), 7.0, dtype=torch.bfloat16, device="cuda")[:, :T].transpose(0, 1) for h in (Hq, Hq, Hkv, Hkv)]
    for places in (ranges, byhead):
        p.out, p.dq, p.dk, p.dv = places
        p.forward(True, 0.1)
        p.backward(True, 0.1)
        torch.cuda.synchronize()
        assert all(np.array_equal(bits_of(t), w) for t, w in zip(places, want))
    used = torch.zeros(T, 20, 80, dtype=torch.bool, device="cuda")
    for a, h in ((6, Hq), (11, Hkv), (15, Hkv)):
        used[:sum(lens), a:a + h, 8:] = True
    assert bool((wide[~used] == 7.0).all())
    other[:sum(lens), 1:1 + Hq, 8:] = 7.0
    assert bool((other == 7.0).all())
    # gradients among the columns of an input are refused: what they span meets it
    p.dq = wide[:, :Hq, :D]
    p.q = wide[:, Hq:2 * Hq, :D]
    with pytest.raises(B.SkipFFNError):
        p.backward(True, 0.1)
