"""Pins for the oracle's attention: closed forms, the library softmax, fp64 autograd and finite differences."""
import numpy as np
import pytest
import torch

from oracle import skipffn_oracle as O


def case(nq, nk, Hq, Hkv, D, seed):
    r = np.random.default_rng(seed)
    return r.standard_normal((nq, Hq, D)), r.standard_normal((nk, Hkv, D)), r.standard_normal((nk, Hkv, D)), r.standard_normal((nq, Hq, D))


def test_closed_forms():
    q, k, v, _ = case(5, 5, 2, 2, 4, 0)
    # queries of zero: the mean of the values seen
    out, P = O.attn_forward_real(0 * q, k, v, True, 0.5)
    for i in range(5):
        assert np.allclose(out[i], v[:i + 1].mean(axis=0), atol=1e-14)
    # the first query sees one key alone
    out, P = O.attn_forward_real(q, k, v, True, 0.5)
    assert np.allclose(out[0], v[0], atol=1e-14) and np.all(P[:, 0, 1:] == 0)
    # weights are a distribution over what is seen
    assert np.allclose(P.sum(axis=2), 1) and np.all(np.triu(P[0], 1) == 0)
    # one more key than queries: every row sees one more
    _, P = O.attn_forward_real(q[:4], k, v, True, 0.5)
    assert np.all(P[:, 0, :2] > 0) and np.all(P[:, 0, 2:] == 0)


def test_rows_that_see_nothing_are_zero_and_carry_no_gradient():
    q, k, v, g = case(5, 3, 2, 1, 4, 1)
    b = O.attn_backward_real(q, k, v, g, True, 0.5)
    assert np.all(b["out"][:2] == 0) and np.all(b["dq"][:2] == 0) and np.all(b["P"][:, :2] == 0)
    assert np.allclose(b["out"][2], v[0, [0, 0]])
    c = O.attn_backward_real(q[2:], k, v, g[2:], True, 0.5)
    assert np.allclose(b["dk"], c["dk"]) and np.allclose(b["dv"], c["dv"])
    # no keys at all
    out, _ = O.attn_forward_real(q, k[:0], v[:0], False, 0.5)
    assert np.all(out == 0)


def test_what_is_not_seen_has_no_part_in_the_weights():
    S = np.array([[0.3, np.nan], [0.1, 0.2]])
    P = O.attn_weights(S, True)
    assert np.all(np.isfinite(P)) and P[0, 0] == 1


@pytest.mark.parametrize("nq,nk,Hq,Hkv,causal", [(7, 7, 4, 2, True), (3, 9, 6, 6, True), (8, 5, 4, 1, True), (6, 11, 2, 1, False)])
def test_against_library_softmax_and_autograd(nq, nk, Hq, Hkv, causal):
    q, k, v, g = case(nq, nk, Hq, Hkv, 8, nq + nk)
    b = O.attn_backward_real(q, k, v, g, causal, 0.35)
    qt, kt, vt = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    rep = Hq // Hkv
    S = torch.einsum("ihd,jhd->hij", qt, kt.repeat_interleave(rep, 1)) * 0.35
    lo = max(nq - nk, 0) if causal else 0                     # rows before it see nothing
    if causal:
        S = S.masked_fill(torch.ones(nq, nk).triu(nk - nq + 1).bool(), -float("inf"))
    out = torch.einsum("hij,jhd->ihd", torch.softmax(S[:, lo:], -1), vt.repeat_interleave(rep, 1))
    assert np.allclose(b["out"][lo:], out.detach().numpy(), atol=1e-13)
    dq, dk, dv = torch.autograd.grad(out, (qt, kt, vt), torch.tensor(g[lo:]))
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert np.allclose(b[name], t.numpy(), atol=1e-12), name


def test_gradients_against_differences():
    q, k, v, g = case(5, 6, 2, 1, 4, 3)
    b = O.attn_backward_real(q, k, v, g, True, 0.5)
    r, eps = np.random.default_rng(4), 1e-6
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        d = r.standard_normal(x.shape)
        def loss(t):
            a = {"dq": q, "dk": k, "dv": v}
            a[name] = x + t * d
            return (O.attn_forward_real(a["dq"], a["dk"], a["dv"], True, 0.5)[0] * g).sum()
        assert np.isclose((loss(eps) - loss(-eps)) / (2 * eps), (b[name] * d).sum(), rtol=1e-6)


def test_one_token_at_a_time_over_a_shared_beginning_is_the_last_row_of_the_whole():
    r = np.random.default_rng(5)
    Hq, Hkv, D = 4, 2, 8
    pk, pv = r.standard_normal((2, 9, Hkv, D))
    sk, sv = r.standard_normal((2, 3, 5, Hkv, D))
    q = r.standard_normal((3, Hq, D))
    lens = [2, 0, 5]
    out, seen = O.attn_decode_real(q, pk, pv, [0, 6, 9], [0, 1, 2], sk, sv, lens, 0.4)
    for i, (a, e) in enumerate([(0, 6), (6, 9), (0, 0)]):     # the third belongs to no group
        k, v = np.concatenate([pk[a:e], sk[i, :lens[i]]]), np.concatenate([pv[a:e], sv[i, :lens[i]]])
        want, _ = O.attn_forward_real(q[i:i + 1], k, v, True, 0.4)
        assert np.allclose(out[i], want[0], atol=1e-14)
        assert np.allclose(seen[i][2].sum(axis=1), 1)
