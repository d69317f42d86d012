"""Norm and rotation of queries and keys through the C ABI against the oracle, element by element within the bounds of
rope_bounds."""
import numpy as np
import pytest
import torch

from attn_bounds import assert_within
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of, to_dev_bf16
from rope_bounds import backward_bounds, forward_bound

pytestmark = pytest.mark.gpu

EPS = 1e-6


def rand(rng, *shape, std=1.0):
    return to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal(shape) * std))


def room(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


class Rope:
    """q, k, v as column ranges of one projection's output, and all that goes with them."""

    def __init__(self, T, Hq, Hkv, D, rot, axes=1, far=0, norm=True, gains=True, pairs=False, seed=0):
        rng = self.rng = np.random.default_rng(seed + T * 7 + D)
        self.T, self.Hq, self.Hkv, self.D, self.rot, self.norm, self.pairs = T, Hq, Hkv, D, rot, norm, pairs
        self.qkv = rand(rng, T, Hq + 2 * Hkv, D, std=1.5)
        self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hkv], self.qkv[:, Hq + Hkv:]
        pos = rng.integers(-50, 5000, (axes, T)) + far
        freq = (500000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))).astype(np.float32)
        axis = rng.integers(0, axes, rot // 2)
        self.pos, self.freq = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(freq).cuda()
        self.axis = None if axes == 1 else axis.tolist()
        self.angle = O.rope_angles(pos, freq, axis)
        self.gq, self.gk = (rand(rng, D, std=0.5) if gains and norm else None for _ in range(2))
        self.flags = (B.FLAG_QK_NORM if norm else 0) | (B.FLAG_ROPE_PAIRS if pairs else 0)
        self.common = dict(axis=self.axis, gain_q=self.gq, gain_k=self.gk, eps=EPS, flags=self.flags)

    def forward(self, q_out, k_out, **more):
        B.skipffn_qk_rope_forward(self.q, self.k, q_out, k_out, self.pos, self.freq, **self.common, **more)

    def want(self, x, gain):
        return O.rope_forward_real(f64_of(x), self.angle, self.pairs, self.norm, None if gain is None else f64_of(gain), EPS)

    def check(self, got, x, gain, what):
        y, n = self.want(x, gain)
        assert_within(f64_of(got), y, forward_bound(y, n, self.rot, self.pairs), what)


SHAPES = [(1, 4, 2, 128, 128), (67, 32, 8, 128, 128), (33, 4, 4, 64, 64), (9, 6, 2, 80, 80), (9, 5, 1, 72, 72), (17, 3, 3, 40, 40), (5, 2, 2, 8, 8),
          (21, 28, 4, 96, 48), (12, 8, 1, 128, 64), (12, 1, 1, 120, 24), (7, 4, 2, 64, 0), (130, 3, 1, 16, 16), (300, 1, 1, 56, 40)]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot", SHAPES)
@pytest.mark.parametrize("norm", [False, True], ids=["bare", "norm"])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("axes", [1, 3])
def test_forward_and_backward(T, Hq, Hkv, D, rot, norm, pairs, axes):
    print(f"rope T={T} heads {Hq}/{Hkv} D={D} rot={rot} norm={norm} pairs={pairs} axes={axes}", flush=True)
    p = Rope(T, Hq, Hkv, D, rot, axes, 0 if axes == 1 else 100000, norm, True, pairs)
    q_out, k_out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out, k_out)
    grads = rand(p.rng, T, Hq, D), rand(p.rng, T, Hkv, D)
    dqkv = torch.full((T, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    dq, dk = dqkv[:, :Hq], dqkv[:, Hq:Hq + Hkv]
    d_gain = [torch.full((D,), 7.0, device="cuda") for _ in range(2)] if norm else [None, None]
    ws = room(B.skipffn_qk_rope_backward_workspace_bytes(T, Hq, Hkv, D))
    B.skipffn_qk_rope_backward(*grads, dq, dk, p.pos, p.freq, q=p.q, k=p.k, d_gain_q=d_gain[0], d_gain_k=d_gain[1], workspace=ws, **p.common)
    torch.cuda.synchronize()
    for name, x, gain, out, g, dx, dg in (("q", p.q, p.gq, q_out, grads[0], dq, d_gain[0]), ("k", p.k, p.gk, k_out, grads[1], dk, d_gain[1])):
        p.check(out, x, gain, name)
        gf = None if gain is None else f64_of(gain)
        want, wg = O.rope_backward_real(f64_of(x), p.angle, pairs, norm, gf, EPS, f64_of(g))
        e, eg = backward_bounds(f64_of(x), norm, gf, EPS, f64_of(g), rot, pairs, want)
        assert_within(f64_of(dx), want, e, f"grad_{name}")
        if norm:
            assert_within(f64_of(dg), wg, eg, f"d_gain_{name}")
    assert bool((dqkv[:, Hq + Hkv:] == 7.0).all())


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 30, -2 ** 31 + 51, 2 ** 31 - 5001])
def test_far_positions(far):
    """Angles of 2^31 radians: the product in 64 bits is off by 2^-22 half turns, four times what nearer positions leave."""
    p = Rope(40, 4, 2, 64, 64, far=far, norm=False)
    q_out, k_out = torch.empty(40, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(40, 2, 64, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out, k_out)
    p.check(q_out, p.q, None, "q")
    p.check(k_out, p.k, None, "k")


def test_gains_are_ones_where_there_are_none():
    p = Rope(19, 4, 2, 128, 128, gains=False)
    a, b = (torch.empty(19, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    p.forward(a, b)
    p.check(a, p.q, None, "q")
    p.common.update(gain_q=torch.ones(128, dtype=torch.bfloat16, device="cuda"))
    c = torch.empty_like(a)
    p.forward(c, b)
    assert np.array_equal(bits_of(a), bits_of(c))


@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("T,D,rot", [(23, 128, 128), (1, 64, 32), (70, 72, 72)])
def test_into_the_rows_of_a_cache(T, D, rot, head_major):
    """Keys and values to rows in no order; tokens of a padded batch, whose row is none, go nowhere, and other rows stay."""
    p = Rope(T, 8, 2, D, rot)
    rows = 2 * T + 5
    shape = (2, 2, rows, D) if head_major else (2, rows, 2, D)
    cache = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    kc, vc = (cache[i].transpose(0, 1) if head_major else cache[i] for i in range(2))
    row = p.rng.permutation(rows)[:T].astype(np.int32)
    row[::5] = [(-1, rows, -2 ** 31, 2 ** 31 - 1)[i % 4] for i in range(len(row[::5]))]
    q_out = torch.empty(T, 8, D, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out, kc, v=p.v, v_out=vc, row=torch.from_numpy(row).cuda())
    p.check(q_out, p.q, p.gq, "q")
    ok = (row >= 0) & (row < rows)
    y, n = p.want(p.k, p.gk)
    assert_within(f64_of(kc)[row[ok]], y[ok], forward_bound(y, n, rot, False)[ok], "k")
    assert np.array_equal(bits_of(vc)[row[ok]], bits_of(p.v)[ok])
    rest = np.ones(rows, dtype=bool)
    rest[row[ok]] = False
    assert np.all(f64_of(kc)[rest] == 7.0) and np.all(f64_of(vc)[rest] == 7.0)


def test_in_place_gives_the_same_bits():
    p = Rope(45, 8, 2, 128, 128, axes=3)
    q_out, k_out = torch.empty(45, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(45, 2, 128, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out, k_out)
    v = bits_of(p.v)
    x = p.q.clone(), p.k.clone()
    p.forward(p.q, p.k)
    assert np.array_equal(bits_of(p.q), bits_of(q_out)) and np.array_equal(bits_of(p.k), bits_of(k_out)) and np.array_equal(bits_of(p.v), v)
    g = rand(p.rng, 45, 12, 128)
    want = torch.empty_like(g)
    args = dict(q=x[0], k=x[1], **p.common)
    B.skipffn_qk_rope_backward(g[:, :8], g[:, 8:10], want[:, :8], want[:, 8:10], p.pos, p.freq, **args)
    B.skipffn_qk_rope_backward(g[:, :8], g[:, 8:10], g[:, :8], g[:, 8:10], p.pos, p.freq, **args)
    assert np.array_equal(bits_of(g[:, :10]), bits_of(want[:, :10]))


def test_gain_gradients_add_up_and_come_alone():
    T = 400
    p = Rope(T, 8, 2, 64, 64)
    g = rand(p.rng, T, 8, 64), rand(p.rng, T, 2, 64)
    dq, dk = torch.empty(T, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 2, 64, dtype=torch.bfloat16, device="cuda")
    ws = room(B.skipffn_qk_rope_backward_workspace_bytes(T, 8, 2, 64))
    a, b = torch.zeros(64, device="cuda"), torch.full((64,), 3.0, device="cuda")
    args = dict(q=p.q, k=p.k, workspace=ws, **{**p.common})
    B.skipffn_qk_rope_backward(*g, dq, dk, p.pos, p.freq, d_gain_q=a, **args)
    args["flags"] |= B.FLAG_DW_ACCUMULATE
    B.skipffn_qk_rope_backward(*g, dq, dk, p.pos, p.freq, d_gain_q=b, **args)
    assert torch.equal(b, a + 3.0)
    # the same bits every time
    c = torch.zeros(64, device="cuda")
    B.skipffn_qk_rope_backward(*g, dq, dk, p.pos, p.freq, d_gain_q=c, **args)
    assert torch.equal(c, a)


def test_no_tokens():
    p = Rope(0, 4, 2, 64, 64)
    e = lambda h: torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda")
    p.forward(e(4), e(2))
    d = [torch.full((64,), 5.0, device="cuda") for _ in range(2)]
    B.skipffn_qk_rope_backward(e(4), e(2), e(4), e(2), p.pos, p.freq, q=p.q, k=p.k, d_gain_q=d[0], d_gain_k=d[1],
                               workspace=room(B.skipffn_qk_rope_backward_workspace_bytes(0, 4, 2, 64)), **p.common)
    assert bool((d[0] == 0).all() and (d[1] == 0).all())


def test_values_that_are_not_finite_stay_in_their_head():
    """Without the norm a pair turns by itself; columns that are not rotated pass as they are; with the norm a head is one."""
    for norm in (False, True):
        p = Rope(6, 4, 2, 64, 32, norm=norm)
        p.q[2, 1, 5] = float("inf")
        p.q[3, 0, 50] = float("nan")
        p.q[4, 2, 60] = float("inf")
        q_out, k_out = torch.empty(6, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 2, 64, dtype=torch.bfloat16, device="cuda")
        p.forward(q_out, k_out)
        bad = ~np.isfinite(f64_of(q_out))
        want = np.zeros_like(bad)
        if norm:
            want[3, 0] = True                            # a NaN makes the whole head one
            assert bad[2, 1, 5] and bad[4, 2, 60]        # infinity times the 0 that an infinite mean leaves
            bad[2, 1] = bad[4, 2] = False
        else:
            want[2, 1, [5, 21]] = want[3, 0, 50] = want[4, 2, 60] = True
            assert f64_of(q_out)[4, 2, 60] == np.inf
        assert np.array_equal(bad, want) and np.isfinite(f64_of(k_out)).all()


def test_offsets_past_32_bits():
    """Rows of a cache of 5 GB."""
    p = Rope(8, 4, 2, 128, 128)
    rows = 2 ** 23 + 77
    cache = torch.zeros(rows, 2, 128, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(rows, 2, 128, dtype=torch.bfloat16, device="cuda")
    row = np.array([0, rows - 1, 2 ** 22 + 3, 2 ** 23, 5, 2 ** 23 + 70, 2 ** 21, 17], dtype=np.int32)
    q_out = torch.empty(8, 4, 128, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out, cache, v=p.v, v_out=vc, row=torch.from_numpy(row).cuda())
    at = torch.from_numpy(row).long().cuda()
    p.check(cache[at], p.k, p.gk, "k")
    assert np.array_equal(bits_of(vc[at]), bits_of(p.v))
    assert int((cache != 0).any(-1).any(-1).sum()) == 8


def test_captured_and_replayed():
    T = 300
    p = Rope(T, 8, 2, 64, 64)
    q_out, k_out = torch.empty(T, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 2, 64, dtype=torch.bfloat16, device="cuda")
    g = rand(p.rng, T, 8, 64), rand(p.rng, T, 2, 64)
    dq, dk = torch.empty_like(q_out), torch.empty_like(k_out)
    d = [torch.zeros(64, device="cuda") for _ in range(2)]
    ws = room(B.skipffn_qk_rope_backward_workspace_bytes(T, 8, 2, 64))

    def work():
        p.forward(q_out, k_out)
        B.skipffn_qk_rope_backward(*g, dq, dk, p.pos, p.freq, q=p.q, k=p.k, d_gain_q=d[0], d_gain_k=d[1], workspace=ws, **p.common)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        p.qkv.copy_(rand(p.rng, T, 12, 64))
        p.pos += 11
        work()
        want = [t.clone() for t in (q_out, k_out, dq, dk, *d)]
        for t in (q_out, k_out, dq, dk, *d):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (q_out, k_out, dq, dk, *d))), turn


# ---- more wavefronts than the chip holds -----------------------------------------------------------------
# Beyond 32 a compute unit a forward wavefront works on three heads one after the other; a backward one goes on through the tokens.
def lanes_of_a_head(D, rot, pairs):
    wide = pairs or rot % 16 == 0                        # slots of 8 columns, otherwise of 4
    return (4 if wide else 8) * (1 if D <= 64 else 2)


def wavefronts(T, heads, D, rot, pairs):
    """Of T tokens where each has one round of heads."""
    lanes, at_once = lanes_of_a_head(D, rot, pairs), 1
    while at_once * 2 * lanes <= 64 and at_once < heads:
        at_once *= 2
    return -(-T // (64 // lanes // at_once)) * -(-heads // at_once)


def chip():
    return torch.cuda.get_device_properties(0).multi_processor_count


MANY = [(1800, 32, 8, 128, 128), (1800, 28, 4, 128, 128), (4300, 10, 2, 72, 72), (8400, 9, 3, 40, 40), (4200, 20, 5, 64, 32), (70001, 1, 1, 8, 8),
        (3000, 6, 6, 96, 0)]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot", MANY)
@pytest.mark.parametrize("norm", [False, True], ids=["bare", "norm"])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "neighbours"])
def test_many_tokens_into_the_rows_of_a_cache(T, Hq, Hkv, D, rot, norm, pairs):
    print(f"many tokens T={T} heads {Hq}/{Hkv} D={D} rot={rot} norm={norm} pairs={pairs}", flush=True)
    assert wavefronts(T, Hq + 2 * Hkv, D, rot, pairs) > 32 * chip()
    p = Rope(T, Hq, Hkv, D, rot, 3 if rot else 1, 1000, norm, True, pairs)
    rows = T + 77
    kc, vc = (torch.full((Hkv, rows, D), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2))
    row = p.rng.permutation(rows)[:T].astype(np.int32)
    row[::5] = [(-1, rows, -2 ** 31, 2 ** 31 - 1)[i % 4] for i in range(len(row[::5]))]
    q_out = torch.full((T, Hq + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    p.forward(q_out[:, :Hq], kc, v=p.v, v_out=vc, row=torch.from_numpy(row).cuda())
    torch.cuda.synchronize()
    p.check(q_out[:, :Hq], p.q, p.gq, "q")
    assert bool((q_out[:, Hq] == 7.0).all())
    ok = (row >= 0) & (row < rows)
    y, n = p.want(p.k, p.gk)
    assert_within(f64_of(kc)[row[ok]], y[ok], forward_bound(y, n, rot, pairs)[ok], "k")
    at = torch.from_numpy(row[ok]).long().cuda()
    assert torch.equal(vc[at].view(torch.int16), p.v[torch.from_numpy(ok).cuda()].view(torch.int16))
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert bool((kc[rest] == 7.0).all() and (vc[rest] == 7.0).all())


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,pairs", [(2100, 28, 4, 128, 128, False), (3100, 9, 2, 72, 72, False), (9000, 7, 2, 64, 64, True)])
def test_many_tokens_in_place(T, Hq, Hkv, D, rot, pairs):
    print(f"many tokens in place T={T} heads {Hq}/{Hkv} D={D}", flush=True)
    assert wavefronts(T, Hq + Hkv, D, rot, pairs) > 32 * chip()
    p = Rope(T, Hq, Hkv, D, rot, pairs=pairs)
    q_out, k_out = (torch.empty(T, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv))
    p.forward(q_out, k_out)
    p.check(q_out, p.q, p.gq, "q")
    p.check(k_out, p.k, p.gk, "k")
    v = p.v.clone()
    p.forward(p.q, p.k)
    assert torch.equal(p.q, q_out) and torch.equal(p.k, k_out) and torch.equal(p.v, v)


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,pairs", [(30000, 16, 4, 16, 16, False), (30001, 16, 4, 16, 8, True), (6000, 8, 2, 72, 72, False), (4001, 12, 3, 128, 64, False)])
@pytest.mark.parametrize("norm", [False, True], ids=["bare", "norm"])
def test_gradients_of_many_tokens(T, Hq, Hkv, D, rot, pairs, norm):
    """Rounds of a wavefront: 4 to 13 (units over the wavefronts of three workgroups a compute unit), which its gains' sums go through."""
    print(f"gradients of many tokens T={T} heads {Hq}/{Hkv} D={D} norm={norm}", flush=True)
    for H in (Hq, Hkv):
        assert wavefronts(T, H, D, rot, pairs) > 3 * 12 * chip() * H / (Hq + Hkv)
    p = Rope(T, Hq, Hkv, D, rot, 1, 0, norm, True, pairs)
    grads = rand(p.rng, T, Hq, D), rand(p.rng, T, Hkv, D)
    ws = room(B.skipffn_qk_rope_backward_workspace_bytes(T, Hq, Hkv, D))
    want = [O.rope_backward_real(f64_of(x), p.angle, pairs, norm, None if gain is None else f64_of(gain), EPS, f64_of(g))
            for x, gain, g in ((p.q, p.gq, grads[0]), (p.k, p.gk, grads[1]))]
    bound = [backward_bounds(f64_of(x), norm, None if gain is None else f64_of(gain), EPS, f64_of(g), rot, pairs, w[0])
             for x, gain, g, w in ((p.q, p.gq, grads[0], want[0]), (p.k, p.gk, grads[1], want[1]))]
    for gains in (True, False) if norm else (False,):
        dqkv = torch.full((T, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
        d_gain = [torch.full((D,), 7.0, device="cuda") for _ in range(2)] if gains else [None, None]
        B.skipffn_qk_rope_backward(*grads, dqkv[:, :Hq], dqkv[:, Hq:Hq + Hkv], p.pos, p.freq, q=p.q, k=p.k, d_gain_q=d_gain[0], d_gain_k=d_gain[1],
                                   workspace=ws, **p.common)
        torch.cuda.synchronize()
        for name, dx, dg, w, e in (("q", dqkv[:, :Hq], d_gain[0], want[0], bound[0]), ("k", dqkv[:, Hq:Hq + Hkv], d_gain[1], want[1], bound[1])):
            assert_within(f64_of(dx), w[0], e[0], f"grad_{name}")
            if gains:
                assert_within(f64_of(dg), w[1], e[1], f"d_gain_{name}")
        assert bool((dqkv[:, Hq + Hkv:] == 7.0).all())
