"""What the rows of a cache receive from single tokens, through the C ABI against the oracle; the attention's own rows bit for bit as
without them.

Bounds: a weight is off by what its score and its row's sum of weights are, each 2^-12 of it (F of attn_bounds); sums are fp32."""
import numpy as np
import pytest
import torch

from attn_bounds import F, assert_within
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of
from test_gpu_attn_decode import CASES, Decode, ints

pytestmark = pytest.mark.gpu


class Weights:
    """What a call adds, beside a Decode: weights of the prefix [Hkv, Tp] and of own rows [n, Hkv, capacity], of 7."""

    def __init__(self, d, by_head=True, most=None):
        self.d = d
        self.most = max(1, int(np.diff(d.off).max()) if d.G else 1) if most is None else most
        self.pw = torch.full((d.Hkv, d.Tp + 3), 7.0, device="cuda")[:, :d.Tp]
        shape = (d.n, d.Hkv, d.cap + 1) if by_head else (d.Hkv, d.n, d.cap + 1)
        sw = torch.full(shape, 7.0, device="cuda")
        self.sw = (sw if by_head else sw.transpose(0, 1))[..., :d.cap]
        self.ws = torch.empty(B.skipffn_attn_decode_weights_workspace_bytes(d.n, d.G, d.Hq, d.Hkv, d.D, d.Tp, d.cap, self.most),
                              dtype=torch.uint8, device="cuda")

    def run(self, scale, flags=0):
        d = self.d
        B.skipffn_attn_decode_weights(d.q, d.pk, d.pv, d.d_seg, d.d_off, d.sk, d.sv, d.d_own, d.out, self.pw, self.sw,
                                      most_shared=self.most, scale=scale, workspace=self.ws, flags=flags)

    def want(self, scale):
        d = self.d
        f = {n: f64_of(getattr(d, n)) for n in ("q", "pk", "pv", "sk", "sv")}
        _, seen = O.attn_decode_real(f["q"], f["pk"], f["pv"], d.seg, d.off, f["sk"], f["sv"], d.own, scale)
        pw, sw = np.full((d.Hkv, d.Tp), np.nan), np.full((d.n, d.Hkv, d.cap), np.nan)
        pw[:, :d.seg[-1]] = 0.0
        group = np.full(d.n, -1)
        for g in range(d.G):
            group[d.off[g]:d.off[g + 1]] = g
        for i, (_, _, P) in enumerate(seen):
            P = P.reshape(d.Hkv, d.Hq // d.Hkv, -1).sum(1)
            rows = d.seg[group[i]:group[i] + 2] if group[i] >= 0 else (0, 0)
            n = rows[1] - rows[0]
            if group[i] < 0 or i - d.off[group[i]] < self.most:
                pw[:, rows[0]:rows[1]] += P[:, :n]
            sw[i, :, :d.own[i]] = P[:, n:]
        return pw, sw

    def check(self, scale, times=1, before=0.0):
        torch.cuda.synchronize()
        for got, want, what in zip((f64_of(self.pw), f64_of(self.sw)), self.want(scale), ("prefix", "own")):
            mine = ~np.isnan(want)
            assert_within(got[mine], before + times * want[mine], 2 * F * times * want[mine] + 2.0 ** -22 * before, what)
            assert np.all(got[~mine] == 7.0), what


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (8, 8, 64), (12, 2, 80), (7, 1, 40), (40, 1, 128), (32, 1, 96), (3, 1, 8)])
@pytest.mark.parametrize("by_head", [True, False], ids=["by head", "by token"])
def test_prefix_and_own_rows(name, Hq, Hkv, D, by_head):
    print(f"decode weights {name} heads {Hq}/{Hkv} D={D} by_head={by_head}", flush=True)
    d = Decode(*CASES[name], Hq, Hkv, D, by_head)
    d.run(D ** -0.5)
    alone = bits_of(d.out)
    d.out.fill_(7.0)
    w = Weights(d, by_head)
    w.run(D ** -0.5)
    w.check(D ** -0.5)
    assert np.array_equal(bits_of(d.out), alone)


def test_sums_over_steps():
    d = Decode((3, 2, 1), (65, 200), (5, 6, 7, 8, 9, 10), 8, 2, 64)
    w = Weights(d)
    for i, n in enumerate(d.own):
        w.sw[i, :, :n] = 2.0
    w.pw[:, :265] = 2.0
    for _ in range(3):
        w.run(0.125, B.FLAG_DW_ACCUMULATE)
    w.check(0.125, times=3, before=2.0)


def test_sequences_past_the_bound_add_nothing_to_the_prefix():
    d = Decode((13, 2, 1), (300, 200), tuple(range(1, 17)), 8, 2, 64)
    d.run(0.125)
    alone = bits_of(d.out)
    w = Weights(d, most=5)
    w.run(0.125)
    w.check(0.125)
    assert np.array_equal(bits_of(d.out), alone)


def test_prefix_or_own_rows_alone():
    d = Decode((2, 3, 0), (700, 65), (4, 5, 6, 7, 8), 8, 2, 128)
    w = Weights(d)
    sizes = (d.n, d.G, 8, 2, 128)
    ws = torch.empty(B.skipffn_attn_decode_weights_workspace_bytes(*sizes, d.Tp, 0, 3), dtype=torch.uint8, device="cuda")
    B.skipffn_attn_decode_weights(d.q, d.pk, d.pv, d.d_seg, d.d_off, None, None, None, d.out, w.pw, None, most_shared=3, scale=0.1, workspace=ws)
    own, d.own = d.own, [0] * d.n
    torch.cuda.synchronize()
    want = w.want(0.1)[0][:, :765]
    assert_within(f64_of(w.pw)[:, :765], want, 2 * F * want, "prefix")
    ws = torch.empty(B.skipffn_attn_decode_weights_workspace_bytes(d.n, 0, 8, 2, 128, 0, d.cap, 0), dtype=torch.uint8, device="cuda")
    B.skipffn_attn_decode_weights(d.q, None, None, None, None, d.sk, d.sv, d.d_own, d.out, None, w.sw, scale=0.1, workspace=ws)
    d.own, d.off = own, np.array([0, 0, 0])
    torch.cuda.synchronize()
    want = w.want(0.1)[1]
    mine = ~np.isnan(want)
    assert_within(f64_of(w.sw)[mine], want[mine], 2 * F * want[mine], "own")


def test_no_sequences():
    """A prefix that nobody reads: its rows receive 0, or nothing more."""
    d = Decode((1, 0), (50,), (3,), 4, 2, 64)
    w = Weights(d)
    e = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    for flags, want in ((B.FLAG_DW_ACCUMULATE, 7.0), (0, 0.0)):
        B.skipffn_attn_decode_weights(e, d.pk, d.pv, d.d_seg, ints([0, 0]), None, None, None, e, w.pw, None, scale=0.1, workspace=w.ws, flags=flags)
        assert bool((w.pw[:, :50] == want).all() and (w.pw[:, 50:] == 7.0).all())


def test_what_is_not_finite_stays_with_who_sees_it():
    d = Decode((2, 2, 1), (100, 70), (5, 6, 7, 8, 9), 4, 2, 64)
    d.sk[1, 3, 0, 5] = float("nan")                      # head 0 of sequence 1, in group 0
    w = Weights(d)
    w.run(0.125)
    torch.cuda.synchronize()
    pw, sw = f64_of(w.pw), f64_of(w.sw)
    assert np.isnan(pw[0, :100]).all() and np.isfinite(pw[1]).all() and np.isfinite(pw[0, 100:]).all()
    assert np.isnan(sw[1, 0, :6]).all() and np.isfinite(sw[1, 1]).all() and np.isfinite(sw[[0, 2, 3, 4]]).all()


def test_captured_and_replayed():
    d = Decode((1, 2, 0), (5000, 3001), (70, 0, 900), 8, 2, 64)
    w = Weights(d)
    w.run(0.125)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.run(0.125, B.FLAG_DW_ACCUMULATE)
    for turn in range(3):
        d.q.mul_(-1.5 if turn else 1.0)
        w.run(0.125)
        want = [2 * w.pw, 2 * w.sw, d.out.clone()]
        d.out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        first, second = w.pw[:, :8001], want[0][:, :8001]
        assert torch.equal(first, second) and torch.equal(d.out, want[2]), turn
        assert all(torch.equal(w.sw[i, :, :n], want[1][i, :, :n]) for i, n in enumerate(d.own)), turn


@pytest.mark.parametrize("prefix", [(900, 333), (3001, 3999), (5003, 2 ** 13)], ids=["few rows", "rows for the chip's half", "many rows"])
@pytest.mark.parametrize("Hq", [8, 16, 32])              # of 8 key/value heads; products of a row 20 to 84
def test_few_and_many_rows_with_few_and_many_products(prefix, Hq):
    print(f"decode weights prefix {prefix} heads {Hq}", flush=True)
    d = Decode((20, 21, 2), prefix, tuple(i * 5 % 37 for i in range(43)), Hq, 8, 40, True)
    d.run(0.2)
    alone = bits_of(d.out)
    w = Weights(d)
    w.run(0.2)
    w.check(0.2)
    assert np.array_equal(bits_of(d.out), alone)
    w.run(0.2, B.FLAG_DW_ACCUMULATE)
    w.check(0.2, times=2)
    short = Weights(d, most=9)                           # those past the ninth of a group add nothing to its prefix
    short.run(0.2)
    short.check(0.2)


def test_products_past_32_bits():
    """16 sequences on one prefix of 2^20 rows: 2^29 products of a head of the cache, 2^31 in all."""
    n, Hq, Hkv, D, Tp = 16, 128, 2, 8, 2 ** 20
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = rand(n, Hq, D), rand(Tp, Hkv, D), rand(Tp, Hkv, D)
    out, pw = torch.empty_like(q), torch.zeros(Hkv, Tp, device="cuda")
    ws = torch.empty(B.skipffn_attn_decode_weights_workspace_bytes(n, 1, Hq, Hkv, D, Tp, 0, n), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 2 ** 33
    B.skipffn_attn_decode_weights(q, k, v, ints([0, Tp]), ints([0, n]), None, None, None, out, pw, None, most_shared=n, scale=0.4, workspace=ws)
    torch.cuda.synchronize()
    for h in range(Hkv):
        want = torch.zeros(Tp, dtype=torch.float64, device="cuda")
        for i in range(n):
            x = (q[i, h * 64:(h + 1) * 64].double() @ k[:, h].double().T) * 0.4
            want += torch.softmax(x, -1).sum(0)
        assert_within(f64_of(pw[h]), want.cpu().numpy(), 2 * F * want.cpu().numpy(), f"head {h}")
