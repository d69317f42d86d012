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
