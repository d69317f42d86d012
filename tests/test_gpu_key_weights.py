"""What the keys of packed prompts receive, through the C ABI against the oracle: the attention's own log-sum-exp, then the weights.

Bounds: a weight is off by what its score and its row's log-sum-exp are, each 2^-12 of it (F of attn_bounds); sums are fp32."""
import numpy as np
import pytest
import torch

from attn_bounds import F, assert_within
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import f64_of, to_dev_bf16

pytestmark = pytest.mark.gpu

BEHIND = 3           # rows behind the last sequence, of NaN


def offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()


def room(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


class Prompt:
    def __init__(self, nq, nk, Hq, Hkv, D, seed=0, head_major=False):
        rng = np.random.default_rng(seed + sum(nq) + D)
        self.nq, self.nk, self.Hq, self.Hkv, self.D = nq, nk, Hq, Hkv, D
        self.T, self.Tk = sum(nq) + BEHIND, sum(nk) + BEHIND
        self.q, self.k, self.v = (self.rows(rng, T, H) for T, H in ((self.T, Hq), (self.Tk, Hkv), (self.Tk, Hkv)))
        if head_major:
            self.k = self.k.transpose(0, 1).contiguous().transpose(0, 1)
        self.seg_q, self.seg_k = offsets(nq), offsets(nk)
        self.saved = room(B.skipffn_attn_saved_bytes(self.T, Hq))
        self.sizes = (self.T, self.Tk, len(nq), Hq, Hkv, D)
        self.w = torch.full((Hkv, self.Tk + 2), 7.0, device="cuda")[:, :self.Tk]

    def rows(self, rng, T, H):
        x = rng.standard_normal((T, H, self.D))
        x[T - BEHIND:] = np.nan
        return to_dev_bf16(O.f64_to_bf16_bits(x))

    def attend(self, causal, scale):
        out = torch.empty_like(self.q)
        B.skipffn_attn_forward(self.q, self.k, self.v, out, self.seg_q, self.seg_k, causal=causal, scale=scale, saved=self.saved,
                               workspace=room(B.skipffn_attn_forward_workspace_bytes(*self.sizes)))

    def receive(self, causal, scale, last=None, flags=0):
        B.skipffn_attn_key_weights(self.q, self.k, self.seg_q, self.seg_k, self.saved, self.w, causal=causal, scale=scale, last=last,
                                   workspace=room(B.skipffn_attn_key_weights_workspace_bytes(*self.sizes, last)), flags=flags)

    def check(self, causal, scale, last=None, times=1, before=0.0):
        torch.cuda.synchronize()
        q, k, w = f64_of(self.q), f64_of(self.k), f64_of(self.w)
        aq = ak = 0
        for s, (nq, nk) in enumerate(zip(self.nq, self.nk)):
            want = O.key_weights_real(q[aq:aq + nq], k[ak:ak + nk], causal, scale, last)
            assert_within(w[:, ak:ak + nk], before + times * want, 2 * F * times * want + 2.0 ** -22 * before, f"sequence {s}")
            aq, ak = aq + nq, ak + nk
        assert np.all(w[:, ak:] == 7.0)


LENGTHS = [((1,), (1,)), ((31, 0, 33, 64), (31, 0, 33, 64)), ((129, 65, 1, 300), (129, 65, 1, 300)), ((40, 7), (333, 7)), ((50, 64, 3), (20, 63, 0)),
           ((5, 0, 9), (0, 70, 129)), ((130,), (1000,)), ((257,), (513,))]


@pytest.mark.parametrize("nq,nk", LENGTHS, ids=str)
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 128), (3, 3, 64), (6, 2, 80), (5, 1, 40), (2, 2, 8), (28, 4, 96), (3, 1, 72)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("last", [None, 1, 50])
def test_packed_sequences(nq, nk, Hq, Hkv, D, causal, last):
    print(f"key weights {nq} over {nk} heads {Hq}/{Hkv} D={D} causal={causal} last={last}", flush=True)
    p = Prompt(nq, nk, Hq, Hkv, D, head_major=D == 128)
    p.attend(causal, D ** -0.5)
    p.receive(causal, D ** -0.5, last)
    p.check(causal, D ** -0.5, last)


def test_many_sequences():
    """More sequences than lanes: pieces go sequence by sequence."""
    lens = [1 + i * 7 % 90 for i in range(100)]
    p = Prompt(lens, lens, 2, 1, 64)
    p.attend(True, 0.1)
    p.receive(True, 0.1)
    p.check(True, 0.1)


@pytest.mark.parametrize("last", [None, 70])
def test_queries_in_parts(last):
    """Few keys and many queries: parts, whose sums a second kernel adds; the same bits every time."""
    p = Prompt((1500, 700), (1500, 700), 16, 2, 64)
    assert B.skipffn_attn_key_weights_workspace_bytes(*p.sizes, last) > 0
    p.attend(True, 0.125)
    p.receive(True, 0.125, last)
    p.check(True, 0.125, last)
    first = p.w.clone()
    p.w.fill_(7.0)
    p.receive(True, 0.125, last)
    assert torch.equal(first, p.w)


def test_sums_over_calls():
    p = Prompt((300, 20), (300, 20), 4, 2, 64)
    p.attend(True, 0.125)
    p.w[:, :320] = 2.0
    for _ in range(3):
        p.receive(True, 0.125, flags=B.FLAG_DW_ACCUMULATE)
    p.check(True, 0.125, times=3, before=2.0)


def test_no_query_counts():
    p = Prompt((30,), (30,), 2, 2, 64)
    p.saved.fill_(0xFF)                                  # not read
    p.receive(True, 0.125, 0)
    assert bool((p.w[:, :30] == 0).all() and (p.w[:, 30:] == 7.0).all())
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    p.w.fill_(7.0)
    B.skipffn_attn_key_weights(e, p.k, zero, p.seg_k, p.saved[:0], p.w, causal=False,
                               workspace=room(B.skipffn_attn_key_weights_workspace_bytes(0, p.Tk, 1, 2, 2, 64)))
    assert bool((p.w[:, :30] == 0).all() and (p.w[:, 30:] == 7.0).all())


def test_queries_that_repeat():
    """A token stride of 0: every query of a head is the same row, and rows past the sequence's end read it too."""
    p = Prompt((70,), (70,), 4, 2, 64)
    p.q = p.q[:1].expand(p.T, 4, 64)
    p.attend(True, 0.125)
    p.receive(True, 0.125)
    p.check(True, 0.125)


@pytest.mark.parametrize("what", ["key", "query", "infinite"])
def test_what_is_not_finite_reaches_what_its_queries_see(what):
    p = Prompt((100, 50), (100, 50), 2, 1, 64)
    if what == "key":
        p.k[60, 0, 3] = float("nan")                     # every query from 60 on has no finite log-sum-exp
        bad = range(0, 100)
    elif what == "query":
        p.q[20, 1, 5] = float("nan")                     # sees the keys 0 .. 20
        bad = range(0, 21)
    else:
        # one query all of whose scores are minus infinity: 0 / 0 at the keys it sees
        p.q[20, 1] = 0.0
        p.q[20, 1, 5] = float("-inf")
        p.k[:21, 0, 5] = 1.0
        bad = range(0, 21)
    p.attend(True, 0.125)
    p.receive(True, 0.125)
    got = torch.isnan(p.w[0]).nonzero()[:, 0].tolist()
    assert got == list(bad)


def test_captured_and_replayed():
    p = Prompt((900,), (900,), 8, 1, 64)
    ws = room(B.skipffn_attn_key_weights_workspace_bytes(*p.sizes))
    assert ws.numel() > 16
    p.attend(True, 0.125)

    def work():
        B.skipffn_attn_key_weights(p.q, p.k, p.seg_q, p.seg_k, p.saved, p.w, causal=True, scale=0.125, workspace=ws)
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        p.q.copy_(p.rows(np.random.default_rng(turn), p.T, 8))
        p.attend(True, 0.125)
        work()
        want = p.w.clone()
        p.w.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.w, want), turn


def test_offsets_past_32_bits():
    """Queries and keys of 2^20 elements a token, 2^32 in all, and heads of weights 2^31 elements apart."""
    T, H, K, D = 4200, 2, 2, 8
    big = torch.zeros(T * 2 ** 20, dtype=torch.bfloat16, device="cuda").view(T, 2 ** 20)
    p = Prompt((4200 - BEHIND,), (4200 - BEHIND,), H, K, D)
    q, k = big[:, -H * D:].view(T, H, D), big[:, :K * D].view(T, K, D)
    q.copy_(p.q)
    k.copy_(p.k)
    p.q, p.k = q, k
    p.w = torch.full((2 ** 31 + T,), 7.0, device="cuda").as_strided((K, T), (2 ** 31, 1))
    p.attend(True, 0.35)
    p.receive(True, 0.35)
    p.check(True, 0.35)
