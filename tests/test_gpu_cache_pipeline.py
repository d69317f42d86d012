"""The operators around attention in the order in which a program has them: norm and rotation into the cache, attention, what the keys
receive, eviction, single tokens with weights, eviction of their own rows; and the gradients back through the rotation.  Each stage is checked against the
oracle fed with what the GPU stage before it produced.  Then what holds for each of them: buffers of exactly the sizes asked for, streams."""
import numpy as np
import pytest
import torch

from attn_bounds import F, assert_within, grad_bounds, out_bound
from oracle import skipffn_oracle as O
from paper_2503_21817_amd import binding as B
from helpers import bits_of, f64_of, to_dev_bf16
from rope_bounds import backward_bounds, forward_bound
from test_gpu_guard_bytes import Guarded

pytestmark = pytest.mark.gpu

HQ, HKV, D, EPS = 8, 2, 64, 1e-6


def room(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def ints(v):
    return torch.tensor(np.asarray(v, dtype=np.int32)).cuda()


def rand(rng, *shape, std=1.0):
    return to_dev_bf16(O.f64_to_bf16_bits(rng.standard_normal(shape) * std))


def slices(lens):
    at = np.concatenate([[0], np.cumsum(lens)])
    return [slice(a, b) for a, b in zip(at[:-1], at[1:])]


class Rotation:
    """Frequencies, axes (time, row, column) and gains of a layer."""

    def __init__(self, rng):
        self.freq = (10000.0 ** (-np.arange(D // 2) * 2 / D)).astype(np.float32)
        self.axis = [0 if j < 8 else 1 + j % 2 for j in range(D // 2)]
        self.gq, self.gk = rand(rng, D, std=0.3) + 1, rand(rng, D, std=0.3) + 1
        self.args = dict(axis=self.axis, gain_q=self.gq, gain_k=self.gk, eps=EPS, flags=B.FLAG_QK_NORM)
        self.inv_freq = torch.from_numpy(self.freq).cuda()

    def check(self, got, x, pos, gain, what):
        y, n = O.rope_forward_real(f64_of(x), O.rope_angles(pos, self.freq, self.axis), False, True, f64_of(gain), EPS)
        assert_within(f64_of(got), y, forward_bound(y, n, D, False), what)


def positions(lens):
    return np.concatenate([np.stack([np.arange(n) // 40, np.arange(n) // 8, np.arange(n) % 8]) for n in lens], 1)


def test_prefill_eviction_and_single_tokens():
    rng = np.random.default_rng(77)
    lens, questions, budget = (300, 41, 120), (3, 1, 2), 64
    T, n, cap, scale = sum(lens), sum(questions), 24, D ** -0.5
    print(f"cache pipeline lens={lens} questions={questions}", flush=True)
    rot = Rotation(rng)
    qkv = rand(rng, T, HQ + 2 * HKV, D)
    q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
    pos, seg = positions(lens), ints(np.concatenate([[0], np.cumsum(lens)]))
    cache = torch.full((2, HKV, T + 9, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ck, cv = (c.transpose(0, 1) for c in cache)
    q1 = torch.empty(T, HQ, D, dtype=torch.bfloat16, device="cuda")
    B.skipffn_qk_rope_forward(q, k, q1, ck, ints(pos), rot.inv_freq, v=v, v_out=cv, row=torch.arange(T, dtype=torch.int32, device="cuda"), **rot.args)
    sizes = (T, T, len(lens), HQ, HKV, D)
    out, saved = torch.empty_like(q1), room(B.skipffn_attn_saved_bytes(T, HQ))
    B.skipffn_attn_forward(q1, ck[:T], cv[:T], out, seg, saved=saved, workspace=room(B.skipffn_attn_forward_workspace_bytes(*sizes)))
    w = torch.zeros(HKV, T, device="cuda")
    B.skipffn_attn_key_weights(q1, ck[:T], seg, None, saved, w, workspace=room(B.skipffn_attn_key_weights_workspace_bytes(*sizes)))
    # each head keeps rows of its own
    Tp = len(lens) * budget
    small = torch.full((2, HKV, Tp, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    pk, pv = (c.transpose(0, 1) for c in small)
    pw, keep, pseg = torch.zeros(HKV, Tp, device="cuda"), torch.zeros(HKV, Tp, dtype=torch.int32, device="cuda"), torch.zeros_like(seg)
    B.skipffn_kv_evict(ck[:T], cv[:T], w, seg, budget, pk, pv, pw, keep, pseg, first=2, recent=16)
    torch.cuda.synchronize()
    rot.check(q1, q, pos, rot.gq, "q")
    rot.check(ck[:T], k, pos, rot.gk, "k")
    assert np.array_equal(bits_of(cv[:T]), bits_of(v)) and bool(torch.isnan(cache[:, :, T:]).all())
    f = {x: f64_of(t) for x, t in (("q", q1), ("k", ck[:T]), ("v", cv[:T]), ("out", out), ("w", w))}
    for s in slices(lens):
        want, P = O.attn_forward_real(f["q"][s], f["k"][s], f["v"][s], True, scale)
        assert_within(f["out"][s], want, out_bound(P, f["v"][s], want), "attention")
        want = O.key_weights_real(f["q"][s], f["k"][s], True, scale)
        assert_within(f["w"][:, s], want, 2 * F * want, "weights")
    kept = [min(m, budget) for m in lens]
    assert pseg.tolist() == np.concatenate([[0], np.cumsum(kept)]).tolist()
    for s, (src, dst) in enumerate(zip(slices(lens), slices(kept))):
        for h in range(HKV):
            rows = O.evict_choice(f["w"][h, src], budget, 2, 16)
            assert np.array_equal(keep[h, dst].cpu().numpy(), rows)
            for a, b in ((ck, pk), (cv, pv)):
                assert np.array_equal(bits_of(b[dst, h]), bits_of(a[src, h])[rows])
            assert np.array_equal(pw[h, dst].cpu().numpy(), w[h, src].cpu().numpy()[rows])

    # answers: own rows of every sequence in a cache [head][sequence][row][column], which the rotation writes and the attention reads
    own = torch.full((2, HKV, n, cap, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sk, sv = (c.permute(1, 2, 0, 3) for c in own)
    sw = torch.zeros(HKV, n, cap, device="cuda").transpose(0, 1)
    own_len = ints([0] * n)
    off, shared = np.concatenate([[0], np.cumsum(questions)]), max(questions)
    ws = room(B.skipffn_attn_decode_weights_workspace_bytes(n, len(lens), HQ, HKV, D, Tp, cap, shared))
    base, group = torch.arange(n, dtype=torch.int32, device="cuda") * cap, np.repeat(np.arange(len(lens)), questions)
    segs = pseg.cpu().numpy()
    for step in range(5):
        new = rand(rng, n, HQ + 2 * HKV, D)
        at = np.stack([np.asarray(lens)[group] + step] * 3)
        q2, answer = torch.empty(n, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, HQ, D, dtype=torch.bfloat16, device="cuda")
        flat = [c.reshape(HKV, n * cap, D).transpose(0, 1) for c in own]
        B.skipffn_qk_rope_forward(new[:, :HQ], new[:, HQ:HQ + HKV], q2, flat[0], ints(at), rot.inv_freq, v=new[:, HQ + HKV:], v_out=flat[1],
                                  row=base + own_len, **rot.args)
        own_len += 1
        before = f64_of(pw), f64_of(sw)
        B.skipffn_attn_decode_weights(q2, pk, pv, pseg, ints(off), sk, sv, own_len, answer, pw, sw, most_shared=shared, workspace=ws,
                                      flags=B.FLAG_DW_ACCUMULATE)
        torch.cuda.synchronize()
        rot.check(sk[:, step], new[:, HQ:HQ + HKV], at, rot.gk, f"k of step {step}")
        want, seen = O.attn_decode_real(f64_of(q2), f64_of(pk), f64_of(pv), segs, off, f64_of(sk), f64_of(sv), [step + 1] * n, scale)
        add = [np.zeros_like(before[0]), np.zeros_like(before[1])]
        for i, (_, vi, P) in enumerate(seen):
            assert_within(f64_of(answer)[i:i + 1], want[i:i + 1], out_bound(P[:, None], vi, want[i:i + 1]), f"answer {i}, step {step}")
            P = P.reshape(HKV, HQ // HKV, -1).sum(1)
            m = segs[group[i] + 1] - segs[group[i]]
            add[0][:, segs[group[i]]:segs[group[i] + 1]] += P[:, :m]
            add[1][i, :, :step + 1] = P[:, m:]
        for got, b, a in zip((f64_of(pw), f64_of(sw)), before, add):
            assert_within(got, b + a, 2 * F * a + 2.0 ** -22 * b, f"weights of step {step}")
    # own rows down to 3, the last one always among them
    fresh = torch.full_like(own, float("nan"))
    fk, fv = (c.permute(1, 2, 0, 3) for c in fresh)
    fw, keep, left = torch.zeros_like(sw), torch.zeros(n, HKV, cap, dtype=torch.int32, device="cuda"), torch.zeros_like(own_len)
    B.skipffn_kv_evict(sk, sv, sw, own_len, 3, fk, fv, fw, keep, left, recent=1)
    torch.cuda.synchronize()
    assert left.tolist() == [3] * n
    for i in range(n):
        for h in range(HKV):
            rows = O.evict_choice(f64_of(sw)[i, h, :5], 3, 0, 1)
            assert rows[-1] == 4 and np.array_equal(keep[i, h, :3].cpu().numpy(), rows)
            assert np.array_equal(bits_of(fk[i, :3, h]), bits_of(sk[i, :, h])[rows]) and np.array_equal(bits_of(fv[i, :3, h]), bits_of(sv[i, :, h])[rows])


def test_training_step_through_the_rotation():
    rng = np.random.default_rng(78)
    lens, scale = (130, 33), D ** -0.5
    T = sum(lens)
    rot, pos, seg = Rotation(rng), positions(lens), ints(np.concatenate([[0], np.cumsum(lens)]))
    qkv = rand(rng, T, HQ + 2 * HKV, D)
    q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
    q1, k1 = torch.empty(T, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, HKV, D, dtype=torch.bfloat16, device="cuda")
    B.skipffn_qk_rope_forward(q, k, q1, k1, ints(pos), rot.inv_freq, **rot.args)
    sizes = (T, T, len(lens), HQ, HKV, D)
    out, saved = torch.empty_like(q1), room(B.skipffn_attn_saved_bytes(T, HQ))
    B.skipffn_attn_forward(q1, k1, v, out, seg, saved=saved, workspace=room(B.skipffn_attn_forward_workspace_bytes(*sizes)))
    g, dqkv = rand(rng, T, HQ, D), torch.empty_like(qkv)
    dq, dk, dv = dqkv[:, :HQ], dqkv[:, HQ:HQ + HKV], dqkv[:, HQ + HKV:]
    B.skipffn_attn_backward(q1, k1, v, out, g, seg, None, saved, dq, dk, dv, workspace=room(B.skipffn_attn_backward_workspace_bytes(*sizes)))
    g1 = {"q": f64_of(dq), "k": f64_of(dk)}
    d_gain = [torch.empty(D, device="cuda") for _ in range(2)]
    B.skipffn_qk_rope_backward(dq, dk, dq, dk, ints(pos), rot.inv_freq, q=q, k=k, d_gain_q=d_gain[0], d_gain_k=d_gain[1],
                               workspace=room(B.skipffn_qk_rope_backward_workspace_bytes(T, HQ, HKV, D)), **rot.args)
    torch.cuda.synchronize()
    rot.check(q1, q, pos, rot.gq, "q")
    f = {x: f64_of(t) for x, t in (("q", q1), ("k", k1), ("v", v), ("dv", dv))}
    for s in slices(lens):
        b = O.attn_backward_real(f["q"][s], f["k"][s], f["v"][s], f64_of(g)[s], True, scale)
        e = grad_bounds(f["q"][s], f["k"][s], f["v"][s], f64_of(g)[s], scale, b)
        for name, got in (("dq", g1["q"][s]), ("dk", g1["k"][s]), ("dv", f["dv"][s])):
            assert_within(got, b[name], e[name], name)
    angle = O.rope_angles(pos, rot.freq, rot.axis)
    for name, x, gain, got, dg in (("q", q, rot.gq, dq, d_gain[0]), ("k", k, rot.gk, dk, d_gain[1])):
        want, wg = O.rope_backward_real(f64_of(x), angle, False, True, f64_of(gain), EPS, g1[name])
        e, eg = backward_bounds(f64_of(x), True, f64_of(gain), EPS, g1[name], D, False, want)
        assert_within(f64_of(got), want, e, f"grad_{name}")
        assert_within(f64_of(dg), wg, eg, f"d_gain_{name}")


# ---- buffers of exactly the sizes asked for ---------------------------------------------------------------
def guarded(nbytes, name, kept):
    g = Guarded(nbytes, name)
    kept.append(g)
    return g


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 1, 1, 8), (77, 12, 4, 72), (600, 32, 8, 128)])
def test_rotation_stays_inside_its_buffers(T, Hq, Hkv, d):
    kept, rng = [], np.random.default_rng(5)
    bf = lambda n, *s: guarded(2 * int(np.prod(s)), n, kept).typed(torch.bfloat16, s)
    q, k = rand(rng, T, Hq, d), rand(rng, T, Hkv, d)
    pos, freq = ints(np.arange(T)), torch.rand(d // 2, device="cuda")
    qo, ko, vo = bf("q_out", T, Hq, d), bf("k_out", T + 3, Hkv, d), bf("v_out", T + 3, Hkv, d)
    B.skipffn_qk_rope_forward(q, k, qo, ko, pos, freq, v=k, v_out=vo, row=ints(np.arange(T)[::-1] + 3), flags=B.FLAG_QK_NORM)
    dq, dk = bf("grad_q", T, Hq, d), bf("grad_k", T, Hkv, d)
    gains = [guarded(4 * d, "d_gain", kept).typed(torch.float32, (d,)) for _ in range(2)]
    ws = guarded(B.skipffn_qk_rope_backward_workspace_bytes(T, Hq, Hkv, d), "workspace", kept)
    B.skipffn_qk_rope_backward(q, k, dq, dk, pos, freq, q=q, k=k, d_gain_q=gains[0], d_gain_k=gains[1], workspace=ws.view, flags=B.FLAG_QK_NORM)
    torch.cuda.synchronize()
    for g in kept:
        g.check()
    assert all(bool(torch.isfinite(t.float()).all()) for t in (qo, dq, dk, *gains))


@pytest.mark.parametrize("members,prefix,cap,Hq,Hkv,d", [((1, 2, 0), (33, 200), 9, 4, 2, 64), ((40, 0, 3), (301, 77), 33, 8, 1, 128),
                                                         ((2, 1, 0), (9001, 4000), 130, 8, 8, 72), ((50,), (65,), 1, 40, 1, 8)])
def test_single_tokens_with_weights_stay_inside_their_buffers(members, prefix, cap, Hq, Hkv, d):
    kept, rng = [], np.random.default_rng(6)
    n, Tp = sum(members), sum(prefix)
    f32 = lambda n, *s: guarded(4 * int(np.prod(s)), n, kept).typed(torch.float32, s)
    out = guarded(2 * n * Hq * d, "out", kept).typed(torch.bfloat16, (n, Hq, d))
    pw, sw = f32("prefix weights", Hkv, Tp), f32("own weights", n, Hkv, cap)
    groups = len(prefix)
    off = np.concatenate([[0], np.cumsum(members[:groups])])
    most = int(np.diff(off).max())
    ws = guarded(B.skipffn_attn_decode_weights_workspace_bytes(n, groups, Hq, Hkv, d, Tp, cap, most), "workspace", kept)
    B.skipffn_attn_decode_weights(rand(rng, n, Hq, d), rand(rng, Tp, Hkv, d), rand(rng, Tp, Hkv, d), ints(np.concatenate([[0], np.cumsum(prefix)])),
                                  ints(off), rand(rng, n, cap, Hkv, d), rand(rng, n, cap, Hkv, d), ints([cap] * n), out, pw, sw, most_shared=most,
                                  workspace=ws.view)
    torch.cuda.synchronize()
    for g in kept:
        g.check()
    assert bool(torch.isfinite(out.float()).all())
    # the weights of a token's query heads add up to as many
    total = pw.sum() + sw.sum()
    assert abs(float(total) / (n * Hq) - 1) < 2 * F


@pytest.mark.parametrize("lens,last", [((1,), None), ((257, 64, 3), None), ((700, 900), 50), ((3000,), None)])
def test_key_weights_stay_inside_their_buffers(lens, last):
    kept, rng = [], np.random.default_rng(7)
    T, H, K, d = sum(lens), 16, 2, 128
    q, k = rand(rng, T, H, d), rand(rng, T, K, d)
    seg, sizes = ints(np.concatenate([[0], np.cumsum(lens)])), (T, T, len(lens), H, K, d)
    saved = guarded(B.skipffn_attn_saved_bytes(T, H), "saved", kept)
    B.skipffn_attn_forward(q, k, k, torch.empty_like(q), seg, saved=saved.view, workspace=room(B.skipffn_attn_forward_workspace_bytes(*sizes)))
    w = guarded(4 * K * T, "weights", kept).typed(torch.float32, (K, T))
    ws = guarded(B.skipffn_attn_key_weights_workspace_bytes(*sizes, last), "workspace", kept)
    B.skipffn_attn_key_weights(q, k, seg, None, saved.view, w, last=last, workspace=ws.view if ws.nbytes else None)
    torch.cuda.synchronize()
    for g in kept:
        g.check()
    counted = H * sum(min(n, last or n) for n in lens)
    assert abs(float(w.sum()) / counted - 1) < 2 * F


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("rows", [(1,), (700, 64, 3), (5000,)])
def test_eviction_stays_inside_its_buffers(packed, rows):
    kept, rng = [], np.random.default_rng(8)
    n, K, d, budget = len(rows), 3, 72, 50
    T = sum(rows) if packed else max(rows)
    lead, T_out = (() if packed else (n,)), (sum(min(m, budget) for m in rows) if packed else budget)
    ko, vo = (guarded(2 * int(np.prod((*lead, T_out, K, d))), "rows", kept).typed(torch.bfloat16, (*lead, T_out, K, d)) for _ in range(2))
    wo, keep = (guarded(4 * int(np.prod((*lead, K, T_out))), "per row", kept).typed(t, (*lead, K, T_out)) for t in (torch.float32, torch.int32))
    seg = ints(np.concatenate([[0], np.cumsum(rows)])) if packed else ints(rows)
    so = guarded(4 * seg.numel(), "seg_out", kept).typed(torch.int32, (seg.numel(),))
    B.skipffn_kv_evict(rand(rng, *lead, T, K, d), rand(rng, *lead, T, K, d), torch.rand(*lead, K, T, device="cuda"), seg, budget, ko, vo, wo, keep, so)
    torch.cuda.synchronize()
    for g in kept:
        g.check()
    assert int(so.max()) == (T_out if packed else min(budget, max(rows)))


# ---- streams ---------------------------------------------------------------------------------------------
def test_two_calls_at_once_on_two_streams():
    """Each on a stream and with workspaces of its own: the same bits as one after the other."""
    rng = np.random.default_rng(9)
    T, H, K, d = 3000, 8, 2, 64
    sizes, scale = (T, T, 1, H, K, d), d ** -0.5
    seg, pos, freq = ints([0, T]), ints(np.arange(T)), torch.rand(d // 2, device="cuda")

    class Work:
        def __init__(self):
            self.q, self.k, self.v = rand(rng, T, H, d), rand(rng, T, K, d), rand(rng, T, K, d)
            e = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")
            self.qo, self.ko, self.out, self.dq, self.dk = e(T, H, d), e(T, K, d), e(T, H, d), e(T, H, d), e(T, K, d)
            self.dg, self.w = [e(d, t=torch.float32) for _ in range(2)], e(K, T, t=torch.float32)
            self.kk, self.vv, self.ww, self.keep, self.so = e(500, K, d), e(500, K, d), e(K, 500, t=torch.float32), e(K, 500, t=torch.int32), e(2, t=torch.int32)
            self.pw, self.answer = e(K, 500, t=torch.float32), e(3, H, d)
            self.saved, self.fws = room(B.skipffn_attn_saved_bytes(T, H)), room(B.skipffn_attn_forward_workspace_bytes(*sizes))
            self.kws, self.rws = room(B.skipffn_attn_key_weights_workspace_bytes(*sizes)), room(B.skipffn_qk_rope_backward_workspace_bytes(T, H, K, d))
            self.dws = room(B.skipffn_attn_decode_weights_workspace_bytes(3, 1, H, K, d, 500, 0, 3))

        def run(self):
            B.skipffn_qk_rope_forward(self.q, self.k, self.qo, self.ko, pos, freq, flags=B.FLAG_QK_NORM)
            B.skipffn_attn_forward(self.qo, self.ko, self.v, self.out, seg, saved=self.saved, workspace=self.fws)
            B.skipffn_attn_key_weights(self.qo, self.ko, seg, None, self.saved, self.w, workspace=self.kws)
            B.skipffn_kv_evict(self.ko, self.v, self.w, seg, 500, self.kk, self.vv, self.ww, self.keep, self.so, recent=100)
            B.skipffn_attn_decode_weights(self.qo[:3], self.kk, self.vv, self.so, off, None, None, None, self.answer, self.pw, None, most_shared=3,
                                          workspace=self.dws)
            B.skipffn_qk_rope_backward(self.out, self.ko, self.dq, self.dk, pos, freq, q=self.q, k=self.k, d_gain_q=self.dg[0], d_gain_k=self.dg[1],
                                       workspace=self.rws, flags=B.FLAG_QK_NORM)

        def results(self):
            return [t.clone() for t in (self.qo, self.ko, self.out, self.w, self.kk, self.vv, self.ww, self.keep, self.answer, self.pw, self.dq, self.dk, *self.dg)]

    off = ints([0, 3])
    works = [Work(), Work()]
    for w in works:
        w.run()
    torch.cuda.synchronize()
    want = [w.results() for w in works]
    streams = [torch.cuda.Stream() for _ in works]
    for turn in range(3):
        for w in works:
            for t in (w.qo, w.out, w.w, w.kk, w.answer, w.pw, w.dq):
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(4):
            for w, s in zip(works, streams):
                with torch.cuda.stream(s):
                    w.run()
        torch.cuda.synchronize()
        for w, r in zip(works, want):
            assert all(torch.equal(a, b) for a, b in zip(w.results(), r)), turn
