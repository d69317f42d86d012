"""Attention of single new tokens over a shared prefix and their own rows through the C ABI, against the oracle, element by
element within the bounds of attn_bounds."""
import numpy as np
import pytest
import torch

from attn_bounds import assert_within, out_bound
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of, to_dev_bf16

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v, dtype=np.int32)).cuda()


class Decode:
    """members: sequences of every group, then (last entry) those of none; prefix: rows of every group; own: rows of every
    sequence.  Rows that nobody has hold NaN."""

    def __init__(self, members, prefix, own, Hq, Hkv, D, by_head=True, seed=0):
        rng = np.random.default_rng(seed + sum(prefix) + D)
        self.n, self.G, self.Hq, self.Hkv, self.D = sum(members), len(prefix), Hq, Hkv, D
        assert len(own) == self.n and len(members) == self.G + 1
        self.seg, self.off = np.concatenate([[0], np.cumsum(prefix)]), np.concatenate([[0], np.cumsum(members[:-1])])
        self.own = list(own)
        self.Tp, self.cap = int(self.seg[-1]) + 5, max(own) + 2
        pre = rng.standard_normal((2, self.Tp, Hkv, D))
        pre[:, self.seg[-1]:] = np.nan
        suf = rng.standard_normal((2, self.n, self.cap, Hkv, D))
        for i, n in enumerate(own):
            suf[:, i, n:] = np.nan
        pre, suf = to_dev_bf16(O.f64_to_bf16_bits(pre)), to_dev_bf16(O.f64_to_bf16_bits(suf))
        if by_head:
            pre = pre.transpose(1, 2).contiguous().transpose(1, 2)
            suf = suf.transpose(2, 3).contiguous().transpose(2, 3)
        (self.pk, self.pv), (self.sk, self.sv) = pre, suf
        self.q = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((self.n, Hq, D))))
        self.out = torch.full((self.n, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.d_seg, self.d_off, self.d_own = ints(self.seg), ints(self.off), ints(own)
        self.ws = torch.empty(max(16, B.skipffn_attn_decode_workspace_bytes(self.n, self.G, Hq, Hkv, D, self.Tp, self.cap)),
                              dtype=torch.uint8, device="cuda")

    def run(self, scale):
        B.skipffn_attn_decode(self.q, self.pk, self.pv, self.d_seg, self.d_off, self.sk, self.sv, self.d_own, self.out, scale=scale,
                              workspace=self.ws)

    def check(self, scale):
        torch.cuda.synchronize()
        f = {n: f64_of(getattr(self, n)) for n in ("q", "pk", "pv", "sk", "sv", "out")}
        want, seen = O.attn_decode_real(f["q"], f["pk"], f["pv"], self.seg, self.off, f["sk"], f["sv"], self.own, scale)
        for i, (k, v, P) in enumerate(seen):
            # parts are joined by fp32 weights: F covers them
            assert_within(f["out"][i:i + 1], want[i:i + 1], out_bound(P[:, None], v, want[i:i + 1]), f"sequence {i}")


CASES = {
    "each its own": ((1, 1, 1, 0), (40, 7, 130), (3, 0, 33)),
    "all share": ((5, 0), (300,), (1, 64, 31, 0, 100)),
    "some of none": ((3, 2, 2), (65, 1), (5, 6, 7, 8, 9, 10, 0)),
    "empty group and prefix": ((0, 2, 1, 0), (50, 0, 33), (0, 4, 2)),
    "many": ((19, 41, 3), (257, 900), tuple(range(63))),
    "long": ((1, 2, 0), (5000, 3001), (70, 0, 900)),
    "large groups, short": ((40, 37, 5), (300, 250), tuple(i % 9 for i in range(82))),
    "large groups, one without a prefix": ((33, 70, 0, 2), (0, 3000, 777), tuple(i * 7 % 130 for i in range(105))),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (8, 8, 64), (12, 2, 80), (7, 1, 40), (40, 1, 128), (32, 1, 96), (3, 1, 8)])
@pytest.mark.parametrize("by_head", [True, False], ids=["by head", "by token"])
def test_shared_prefix_and_own_rows(name, Hq, Hkv, D, by_head):
    print(f"decode {name} heads {Hq}/{Hkv} D={D} by_head={by_head}", flush=True)
    d = Decode(*CASES[name], Hq, Hkv, D, by_head)
    d.run(D ** -0.5)
    d.check(D ** -0.5)
    first = bits_of(d.out)
    d.out.fill_(7.0)
    d.run(D ** -0.5)                                     # the same bits again, whatever the workspace holds now
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(d.out), first)


def test_prefix_alone_and_own_rows_alone():
    members, prefix, own = (4, 0), (200,), (9, 0, 40, 1)
    d = Decode(members, prefix, own, 4, 2, 64)
    B.skipffn_attn_decode(d.q, d.pk, d.pv, d.d_seg, d.d_off, None, None, None, d.out, scale=0.2, workspace=d.ws)
    keep, d.own = d.own, [0] * 4
    d.check(0.2)
    d.out.fill_(7.0)
    ws = torch.empty(max(16, B.skipffn_attn_decode_workspace_bytes(4, 0, 4, 2, 64, 0, d.cap)), dtype=torch.uint8, device="cuda")
    B.skipffn_attn_decode(d.q, None, None, None, None, d.sk, d.sv, d.d_own, d.out, scale=0.2, workspace=ws)
    d.own, d.seg = keep, np.array([0, 0])
    d.check(0.2)


def test_lengths_outside_the_capacity_are_clamped():
    d = Decode((2, 0), (50,), (7, 3), 2, 2, 64)
    d.d_own = ints([-4, 3])
    d.run(0.125)
    d.own = [0, 3]
    d.check(0.125)


def test_a_sequence_that_is_not_finite_leaves_the_others_as_they_are():
    """Infinities and NaN among one sequence's own rows, and in the prefix of one group, reach the rows that see them and no others."""
    Hq, Hkv, D = 8, 2, 128
    d = Decode((5, 3, 0), (100, 70), (40, 33, 0, 70, 5, 1, 64, 9), Hq, Hkv, D)
    d.run(D ** -0.5)
    torch.cuda.synchronize()
    clean = bits_of(d.out)
    d.sv[1, 32, 0, 5] = float("inf")
    d.sv[3, 10, 1, 7] = float("nan")
    d.sk[4, 2, 0, 3] = float("nan")
    d.sv[6, 3] = float("-inf")
    d.run(D ** -0.5)
    torch.cuda.synchronize()
    got, f = bits_of(d.out), f64_of(d.out)
    g = Hq // Hkv
    for i in range(d.n):
        for kh in range(Hkv):
            heads = slice(kh * g, (kh + 1) * g)
            hit = {(1, 0): [5], (3, 1): [7], (4, 0): range(D), (6, 0): range(D), (6, 1): range(D)}.get((i, kh), [])
            keep = [c for c in range(D) if c not in hit]
            assert np.array_equal(got[i, heads][:, keep], clean[i, heads][:, keep]), (i, kh)
            assert not np.isfinite(f[i, heads][:, list(hit)]).any()
    assert np.all(f[1, :g, 5] == np.inf) and np.all(f[6] == -np.inf) and np.all(np.isnan(f[3, g:, 7]))
    # a large group of many products
    w = Decode((50, 0), (700,), tuple(3 + i % 40 for i in range(50)), Hq, Hkv, D, seed=1)
    w.run(D ** -0.5)
    torch.cuda.synchronize()
    before = bits_of(w.out)
    w.sv[13, 2, 1, 4] = float("nan")
    w.sv[40, 0, 0, 100] = float("inf")
    w.run(D ** -0.5)
    torch.cuda.synchronize()
    after, hit = bits_of(w.out), np.zeros((50, Hq, D), bool)
    hit[13, g:, 4] = hit[40, :g, 100] = True
    assert np.array_equal(after[~hit], before[~hit]) and not np.isfinite(f64_of(w.out)[hit]).any()
    # the prefix of the second group: the first group's rows keep their bits
    d.pv[150, 1, 9] = float("nan")
    d.run(D ** -0.5)
    torch.cuda.synchronize()
    assert np.array_equal(bits_of(d.out)[:5], got[:5])
    assert np.all(np.isnan(f64_of(d.out)[5:, g:, 9]))


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (4, 4, 128)])
def test_more_sequences_and_groups_than_lanes(Hq, Hkv, D):
    rng = np.random.default_rng(D)
    members = [int(m) for m in rng.integers(0, 4, 130)] + [7]
    prefix = [int(p) for p in rng.integers(0, 70, 130)]
    own = [int(n) for n in rng.integers(0, 50, sum(members))]
    print(f"decode {sum(members)} sequences, 130 groups, heads {Hq}/{Hkv} D={D}", flush=True)
    d = Decode(members, prefix, own, Hq, Hkv, D)
    d.run(D ** -0.5)
    d.check(D ** -0.5)


def test_offsets_past_32_bits():
    """A cache of 2.2 million rows of 8 heads: elements past 2^31, bytes past 2^32, by token and by head."""
    Hkv, D, Tp = 8, 128, 2_200_000
    rng = np.random.default_rng(3)
    rows = rng.standard_normal((2, 300, Hkv, D))
    bits = O.f64_to_bf16_bits(rows)
    for by_head in (False, True):
        kv = [torch.zeros((Hkv, Tp, D) if by_head else (Tp, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        kv = [t.transpose(0, 1) if by_head else t for t in kv]
        for t, b in zip(kv, bits):
            t[Tp - 300:] = to_dev_bf16(b)
        q = to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal((2, 16, D))))
        out = torch.empty(2, 16, D, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(16, B.skipffn_attn_decode_workspace_bytes(2, 1, 16, Hkv, D, Tp, 0)), dtype=torch.uint8, device="cuda")
        B.skipffn_attn_decode(q, kv[0], kv[1], ints([Tp - 300, Tp]), ints([0, 2]), None, None, None, out, workspace=ws)
        torch.cuda.synchronize()
        f = f64_of(q), O.bf16_bits_to_f64(bits)
        for i in range(2):
            want, P = O.attn_forward_real(f[0][i:i + 1], f[1][0], f[1][1], False, D ** -0.5)
            assert_within(f64_of(out)[i:i + 1], want, out_bound(P, f[1][1], want), f"sequence {i}, by_head={by_head}")
        del kv


def test_what_belongs_together_comes_together():
    d = Decode((2, 0), (50,), (7, 3), 2, 2, 64)
    given = [d.q, d.pk, d.pv, d.d_seg, d.d_off, d.sk, d.sv, d.d_own, d.out]
    for missing in (2, 3, 4, 6, 7):
        with pytest.raises(ValueError, match="belongs"):
            B.skipffn_attn_decode(*(None if i == missing else t for i, t in enumerate(given)), workspace=d.ws)
    with pytest.raises(ValueError, match="prefix or own rows"):
        B.skipffn_attn_decode(d.q, *[None] * 7, d.out, workspace=d.ws)
    with pytest.raises(B.SkipFFNError):
        B.skipffn_attn_decode(d.q, *given[1:8], d.q, workspace=d.ws)


def test_queries_and_results_in_column_ranges_and_by_head():
    Hq, Hkv, D = 6, 2, 40
    d = Decode((3, 2, 1), (100, 300), (5, 0, 33, 64, 1, 7), Hq, Hkv, D)
    d.run(0.2)
    torch.cuda.synchronize()
    want = bits_of(d.out)
    fused = torch.full((d.n, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    fused[:, :Hq] = d.q
    wide = torch.full((d.n, Hq + 3, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    byhead = torch.full((Hq, d.n, D), 7.0, dtype=torch.bfloat16, device="cuda")
    byhead.copy_(d.q.transpose(0, 1))
    for q, out in ((fused[:, :Hq], wide[:, 2:2 + Hq, 8:]), (byhead.transpose(0, 1), torch.full_like(byhead, 7.0).transpose(0, 1))):
        d.q, d.out = q, out
        d.run(0.2)
        torch.cuda.synchronize()
        assert np.array_equal(bits_of(out), want)
    wide[:, 2:2 + Hq, 8:] = 7.0
    assert bool((wide == 7.0).all())
