"""Refusals of the operators around attention, on the host before anything is enqueued, and their size queries."""
import ctypes

import pytest

from paper_2503_21817_amd import binding as B
from test_abi_host import FAKE, FAR, ODD, heads

BIG = 1 << 40
FARS = [FAKE + (i << 32) for i in range(16)]


# ---- norm and rotation -------------------------------------------------------------------------------
def rope_fwd(T=64, Hq=4, Hkv=4, D=64, rot=64, axes=1, t=None, pos=FAKE, freq=FAKE, axis=None, gq=None, gk=None, eps=1e-6, row=None, rows=0,
             flags=B.FLAG_QK_NORM, v=False):
    t = {**{i: heads(FAR[i]) for i in range(6)}, **(t or {})}            # q, k, v, then their outputs
    if not v:
        t[2] = t[5] = None
    return B.lib().skipffn_qk_rope_forward(T, Hq, Hkv, D, rot, axes, t[0], t[1], t[2], pos, freq, axis, gq, gk, eps, row, rows, t[3], t[4], t[5],
                                           flags, None)


def rope_bwd(T=64, Hq=4, Hkv=4, D=64, rot=64, axes=1, t=None, pos=FAKE, freq=FAKE, axis=None, gq=None, gk=None, eps=1e-6, dq=FAKE, dk=FAKE + 1024,
             ws=FAKE, ws_bytes=BIG, flags=B.FLAG_QK_NORM):
    t = {**{i: heads(FAR[i]) for i in range(6)}, **(t or {})}            # q, k, the gradients of the outputs, of q, k
    return B.lib().skipffn_qk_rope_backward(T, Hq, Hkv, D, rot, axes, t[0], t[1], t[2], t[3], pos, freq, axis, gq, gk, eps, t[4], t[5], dq, dk,
                                            ws, ws_bytes, flags, None)


@pytest.mark.parametrize("call", [rope_fwd, rope_bwd])
def test_rope_rejects_bad_arguments(call):
    for bad in (dict(T=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(rot=-8), dict(rot=72), dict(axes=0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(pos=None), dict(pos=ODD), dict(freq=None), dict(freq=ODD), dict(gq=ODD), dict(gk=FAKE + 8),
                dict(gq=FAKE, flags=0), dict(gk=FAKE, flags=0), dict(axis=b"\1" * 32), dict(axis=b"\0" * 31 + b"\3", axes=3)):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(D=60, rot=56), dict(D=136, rot=8), dict(rot=20), dict(rot=4), dict(axes=5), dict(T=1 << 30), dict(Hq=65536), dict(Hkv=65536)):
        assert call(**bad) == B.ESHAPE, bad
    for flags in (0x1, 0x4, 0x8, 0x10, 0x80):
        assert call(flags=flags) == B.EUNSUPPORTED
    for i in (0, 1, 3, 4):
        assert call(t={i: None}) == B.EINVAL
        assert call(t={i: heads(None)}) == B.EINVAL
        assert call(t={i: heads(FAR[i] + 8)}) == B.EINVAL
        assert call(t={i: heads(FAR[i], token=260)}) == B.ESHAPE
        assert call(t={i: heads(FAR[i], token=-256)}) == B.EINVAL


def test_rope_forward_refuses_outputs_that_share_memory():
    assert rope_fwd(flags=B.FLAG_DW_ACCUMULATE) == B.EUNSUPPORTED
    assert rope_fwd(t={3: heads(FAR[3], token=128)}) == B.EINVAL         # rows over one another
    # outputs inside inputs, or inside one another
    for o in (3, 4):
        for i in (0, 1):
            if i != o - 3:
                assert rope_fwd(t={o: heads(FAR[i])}) == B.EINVAL
        assert rope_fwd(t={o: heads(FAR[o - 3] + 128)}) == B.EINVAL      # nearly in place
    assert rope_fwd(t={4: heads(FAR[3])}) == B.EINVAL
    assert rope_fwd(v=True, t={5: heads(FAR[1])}) == B.EINVAL and rope_fwd(v=True, t={4: heads(FAR[2])}) == B.EINVAL
    # keys in place, but to other rows
    assert rope_fwd(t={4: heads(FAR[1])}, row=FAKE, rows=64) == B.EINVAL
    # column ranges of one tensor of 12 heads: in place they are apart, one that reaches into the next is not
    fused = lambda at: heads(FAR[0] + at * 128, token=12 * 64)
    assert rope_fwd(t={0: fused(0), 1: fused(4), 3: fused(0), 4: fused(5)}) == B.EINVAL
    assert rope_fwd(t={0: fused(0), 1: fused(4), 3: fused(2), 4: fused(8)}) == B.EINVAL
    assert rope_fwd(t={0: fused(0), 1: fused(4), 3: fused(0), 4: fused(4)}, row=FAKE, rows=64) == B.EINVAL
    # values: both or none; rows: a sensible number
    assert B.lib().skipffn_qk_rope_forward(64, 4, 4, 64, 64, 1, heads(FAR[0]), heads(FAR[1]), heads(FAR[2]), FAKE, FAKE, None, None, None, 1e-6,
                                           None, 0, heads(FAR[3]), heads(FAR[4]), None, 0, None) == B.EINVAL
    assert rope_fwd(row=FAKE, rows=-1) == B.EINVAL and rope_fwd(row=ODD, rows=64) == B.EINVAL and rope_fwd(row=FAKE, rows=1 << 31) == B.ESHAPE
    # no tokens
    none = {i: heads(None) for i in range(6)}
    assert rope_fwd(T=0, t=none, pos=None, freq=None) == B.OK


def test_rope_backward_refuses_what_it_cannot_do():
    assert rope_bwd(flags=0) == B.EINVAL                                  # gain gradients without a norm
    assert rope_bwd(dq=ODD) == B.EINVAL and rope_bwd(dk=FAKE) == B.EINVAL
    need = B.skipffn_qk_rope_backward_workspace_bytes(64, 4, 4, 64)
    assert need >= 2 * 64 * 4
    assert rope_bwd(ws=None) == B.EWORKSPACE and rope_bwd(ws_bytes=need - 1) == B.EWORKSPACE and rope_bwd(ws=ODD) == B.EWORKSPACE
    for o in (4, 5):
        for i in range(4):
            if i != o - 2:
                assert rope_bwd(t={o: heads(FAR[i])}) == B.EINVAL
    assert rope_bwd(t={5: heads(FAR[4])}) == B.EINVAL
    none = {i: heads(None) for i in range(6)}
    assert rope_bwd(T=0, t=none, pos=None, freq=None, dq=None, dk=None) == B.OK
    for bad in ((-1, 4, 4, 64), (1, 0, 4, 64), (1, 4, 4, 0), (1, 4, 4, 256)):
        assert B.skipffn_qk_rope_backward_workspace_bytes(*bad) == 0


def test_rope_refuses_outputs_over_what_other_workgroups_read():
    wide = [FAKE + (i << 42) for i in range(16)]
    many = 1 << 29                                       # tokens: more than a launch takes, the last of the checks, so that nothing is enqueued
    t = {i: heads(wide[i]) for i in range(6)}
    tables = dict(pos=wide[8], freq=wide[9], row=wide[10], gq=wide[11], gk=wide[12])
    fwd = lambda **more: rope_fwd(T=many, rows=many, v=True, **{**dict(t=t), **tables, **more})
    assert fwd() == B.ESHAPE
    size = dict(pos=many * 4, freq=32 * 4, row=many * 4, gq=64 * 2, gk=64 * 2)
    for o in (3, 4, 5):
        end = wide[o] + many * 4 * 64 * 2
        for name, n in size.items():
            assert fwd(**{name: wide[o]}) == B.EINVAL and fwd(**{name: end - 16}) == B.EINVAL and fwd(**{name: end}) == B.ESHAPE, (o, name)
            assert fwd(**{name: wide[o] - n + 16}) == B.EINVAL and fwd(**{name: wide[o] - n}) == B.ESHAPE, (o, name)
    # a column range of rows that the frequencies lie between
    gap = {**t, 3: heads(wide[3], token=4 * 64 + 64)}
    assert fwd(t=gap, freq=wide[3] + 4 * 64 * 2) == B.ESHAPE and fwd(t=gap, freq=wide[3] + 4 * 64 * 2 - 4) == B.EINVAL
    # the gradients; a workspace that is missing is the last of their checks
    del tables["row"]
    bwd = lambda **more: rope_bwd(ws=None, **{**dict(t=t, dq=wide[13], dk=wide[14]), **tables, **more})
    assert bwd() == B.EWORKSPACE
    for o in (4, 5):
        end = wide[o] + 64 * 4 * 64 * 2
        for name in tables:
            assert bwd(**{name: wide[o]}) == B.EINVAL and bwd(**{name: end - 16}) == B.EINVAL and bwd(**{name: end}) == B.EWORKSPACE, (o, name)
        for name in ("dq", "dk"):
            assert bwd(**{name: wide[o] + 64}) == B.EINVAL and bwd(**{name: end}) == B.EWORKSPACE, (o, name)
    # two gains' gradients: none the other's
    assert bwd(dk=wide[13] + 63 * 4) == B.EINVAL and bwd(dq=wide[14] + 4) == B.EINVAL and bwd(dk=wide[13] + 64 * 4) == B.EWORKSPACE
    assert bwd(dq=None) == B.EWORKSPACE and bwd(dk=None) == B.EWORKSPACE
    # nothing is rotated: neither positions nor frequencies are read
    assert fwd(rot=0, pos=wide[3], freq=wide[3]) == B.ESHAPE and bwd(rot=0, pos=wide[4], freq=wide[5]) == B.EWORKSPACE


# ---- what keys receive -------------------------------------------------------------------------------
def key_weights(Tq=64, Tk=64, n=1, Hq=4, Hkv=4, D=64, q=None, k=None, sq=FAKE, sk=None, scale=0.125, saved=FAKE, last=-1, w=FARS[9], w_head=64,
                ws=FAKE, ws_bytes=BIG, flags=0):
    return B.lib().skipffn_attn_key_weights(Tq, Tk, n, Hq, Hkv, D, q or heads(FAR[0]), k or heads(FAR[1]), sq, sk, 1, scale, saved, last, w, w_head,
                                            ws, ws_bytes, flags, None)


def test_key_weights_reject_bad_arguments():
    for bad in (dict(Tq=-1), dict(n=-1), dict(Hq=0), dict(scale=0.0), dict(scale=float("nan")), dict(sq=None), dict(sk=ODD), dict(Tk=63),
                dict(saved=None), dict(saved=ODD), dict(w=None), dict(w=FARS[9] + 2), dict(w_head=63), dict(w_head=-1), dict(q=heads(None)),
                dict(k=heads(FAR[1] + 8)), dict(w=FAR[0] + 1024), dict(w=FAR[1])):
        assert key_weights(**bad) == B.EINVAL, bad
    for bad in (dict(Hq=6), dict(D=60), dict(D=136), dict(n=65536), dict(Tq=1 << 30, Tk=1 << 30), dict(q=heads(FAR[0], token=260)),
                dict(w_head=1 << 44)):
        assert key_weights(**bad) == B.ESHAPE, bad
    for flags in (0x1, 0x4, 0x20, 0x40):
        assert key_weights(flags=flags) == B.EUNSUPPORTED
    assert key_weights(n=0, saved=None) == B.OK and key_weights(Tk=0, sk=FAKE, k=heads(None), w=None, w_head=0) == B.OK
    # few keys and many queries: parts
    need = B.skipffn_attn_key_weights_workspace_bytes(1 << 16, 64, 1, 4, 4, 64)
    assert need >= 2 * 4 * 64 * 4
    big = dict(Tq=1 << 16, sk=FAKE, q=heads(FAR[2]))
    assert key_weights(**big, ws=None) == B.EWORKSPACE and key_weights(**big, ws_bytes=need - 1) == B.EWORKSPACE and key_weights(**big, ws=ODD) == B.EWORKSPACE
    for bad in ((-1, 1, 1, 1, 1, 8), (1, 1, 1, 3, 2, 8), (1, 1, 1, 1, 1, 9)):
        assert B.skipffn_attn_key_weights_workspace_bytes(*bad) == 0
    # a launch has fewer than 2^32 threads: (63 / 256 + 65535) 256 workgroups fit, 257 times as many do not
    lib = B.lib().skipffn_attn_key_weights
    call = lambda H: lib(63, 63, 65535, H, H, 64, heads(FAR[0], H=H), heads(FAR[1], H=H), FAKE, None, 1, 0.125, FAKE, -1, FARS[9], 64, None, 0, 0x80, None)
    assert call(256) == B.EUNSUPPORTED
    many = lambda H: lib(63, 63, 65535, H, H, 64, heads(FAR[0], H=H), heads(FAR[1], H=H), FAKE, None, 1, 0.125, None, -1, FARS[9], 64, None, 0, 0, None)
    assert many(255) == B.EINVAL and many(257) == B.ESHAPE


def test_key_weights_take_all_that_a_launch_holds():
    """(Tk / 256 + n_seq) Hkv < 2^24 is the bound: the parts that the queries are cut into have to fit it, not the call."""
    lib = B.lib().skipffn_attn_key_weights
    for H, T in ((16, (1 << 26) - 128), (1, (1 << 30) - 128), (25, (1 << 30) // 25 - 256)):
        assert (T // 256 + 1) * H < 1 << 24
        need = B.skipffn_attn_key_weights_workspace_bytes(T, T, 1, H, H, 8)
        assert need >= 2 * H * T * 4, (H, T)
        # no saved sums: refused past the shapes
        t = heads(FAR[0], token=8 * H, head=8, H=H), heads(FAR[1], token=8 * H, head=8, H=H)
        assert lib(T, T, 1, H, H, 8, *t, FAKE, None, 1, 0.125, None, -1, FARS[9], T, None, 0, 0, None) == B.EINVAL, (H, T)


def test_key_weights_reject_weights_over_the_offsets():
    # a workgroup would store them while others still find their sequence by these; parts without a workspace: nothing is enqueued
    parts = dict(Tq=1 << 16, q=heads(FAR[2]), ws=None)
    for bad in (dict(w=FAKE, sk=FARS[12]), dict(w=FAKE + 4, sk=FARS[12]), dict(w=FARS[12], sk=FARS[12]), dict(w=FARS[12] + 4, sk=FARS[12])):
        assert key_weights(**parts, **bad) == B.EINVAL, bad
    assert key_weights(**parts, w=FARS[12] + 8, sk=FARS[12]) == B.EWORKSPACE
    assert key_weights(**parts, w=FARS[12] - 64 * 4, w_head=64 + 2, sk=FARS[12]) == B.EWORKSPACE       # between two heads'
    assert key_weights(**parts, w=FARS[12] - 64 * 4, w_head=64 + 1, sk=FARS[12]) == B.EINVAL
    assert key_weights(w=FAKE) == B.EINVAL               # one table for both


# ---- single tokens with weights ------------------------------------------------------------------------
def dec(n=4, G=1, Hq=4, Hkv=4, D=64, Tp=64, cap=64, t=None, seg=FAKE, off=FAKE, ks=1 << 14, vs=1 << 14, lens=FAKE, scale=0.125, most=4, pw=FARS[8],
        pw_head=64, sw=FARS[9], sw_seq=256, sw_head=64, ws=FAKE, ws_bytes=BIG, flags=0):
    t = {**{i: heads(FAR[i]) for i in range(6)}, **(t or {})}      # q, prefix k, v, own k, v, out
    return B.lib().skipffn_attn_decode_weights(n, G, Hq, Hkv, D, Tp, cap, t[0], t[1], t[2], seg, off, t[3], t[4], ks, vs, lens, t[5], scale, most, pw,
                                               pw_head, sw, sw_seq, sw_head, ws, ws_bytes, flags, None)


def test_decode_weights_reject_bad_arguments():
    for bad in (dict(n=-1), dict(G=-1), dict(Tp=-1), dict(cap=-1), dict(scale=0.0), dict(seg=None), dict(off=ODD), dict(lens=None), dict(ks=-8),
                dict(most=-1), dict(most=0), dict(pw=None), dict(pw=FARS[8] + 2), dict(pw_head=63), dict(pw_head=-1), dict(sw=None), dict(sw=FARS[9] + 1),
                dict(sw_head=63), dict(sw_seq=255), dict(sw_seq=-1), dict(sw_head=-64), dict(sw=FARS[8] + 512)):
        assert dec(**bad) == B.EINVAL, bad
    for bad in (dict(Hq=6), dict(D=60), dict(G=65535), dict(n=1 << 30), dict(ks=4), dict(Tp=(1 << 24), pw_head=1 << 25), dict(pw_head=1 << 44),
                dict(cap=1 << 24, ks=1 << 35, vs=1 << 35, sw_head=1 << 25, sw_seq=1 << 28)):
        assert dec(**bad) == B.ESHAPE, bad
    for flags in (0x1, 0x4, 0x20):
        assert dec(flags=flags) == B.EUNSUPPORTED
    for i in range(6):
        assert dec(t={i: heads(None)}) == B.EINVAL
    for i in range(5):
        assert dec(t={5: heads(FAR[i] + 512)}) == B.EINVAL
    need = B.skipffn_attn_decode_weights_workspace_bytes(4, 1, 4, 4, 64, 64, 64, 4)
    assert need >= 4 * 4 * (4 * 64 + 4 * 64) and dec(ws=None) == B.EWORKSPACE and dec(ws_bytes=need - 1) == B.EWORKSPACE
    # sequences inside a head's range
    assert dec(sw_seq=64, sw_head=256, ws=None) == B.EWORKSPACE
    # nothing to do
    assert dec(n=0, flags=B.FLAG_DW_ACCUMULATE) == B.OK and dec(n=0, Tp=0) == B.OK
    assert B.skipffn_attn_decode_weights_workspace_bytes(4, 1, 4, 4, 64, 64, 64, -1) == 0


def test_decode_weights_reject_weights_over_what_other_workgroups_read():
    last = 64 * 4 * 64 * 2 - 4                           # of a tensor of 64 rows, in bytes; q and out have 4
    for i in range(6):                                   # q, prefix k, v, own k, v, out
        for off in (0, 256, 4 * 4 * 64 * 2 - 4 if i in (0, 5) else last):
            for name in ("pw", "sw"):
                assert dec(t={i: heads(FARS[12])}, ws=None, **{name: FARS[12] + off}) == B.EINVAL, (i, off, name)
    for table, n in (("seg", 2), ("off", 2), ("lens", 4)):
        for name in ("pw", "sw"):
            assert dec(ws=None, **{table: FARS[12], name: FARS[12] + 4 * n - 4}) == B.EINVAL, (table, name)
            assert dec(ws=None, **{table: FARS[12], name: FARS[12] + 4 * n}) == B.EWORKSPACE, (table, name)
    # a prefix alone, own rows alone, a prefix that nobody reads
    assert dec(G=0, Tp=0, pw=None, ws=None, sw=FARS[3]) == B.EINVAL and dec(cap=0, sw=None, ws=None, pw=FARS[2] + 64) == B.EINVAL
    assert dec(n=0, cap=0, pw=FARS[1]) == B.EINVAL and dec(n=0, cap=0, pw=FARS[12], off=FARS[12]) == B.EINVAL
    # every sequence's own keys, values and weights in one place of 64 rows of 4 heads: side by side, and a row too early
    k, w = 64 * 4 * 64, 64 * 4
    slab = 2 * k + 2 * w                                 # elements of 2 bytes
    own = {3: heads(FARS[12]), 4: heads(FARS[12] + 2 * k)}
    at = FARS[12] + 4 * k
    assert dec(t=own, ks=slab, vs=slab, sw=at, sw_seq=slab // 2, ws=None) == B.EWORKSPACE
    assert dec(t=own, ks=slab, vs=slab, sw=at - 4, sw_seq=slab // 2, ws=None) == B.EINVAL
    assert dec(t=own, ks=slab, vs=slab, sw=at + 4, sw_seq=slab // 2, ws=None) == B.EINVAL


# ---- eviction ----------------------------------------------------------------------------------------
def evict(n=2, H=4, D=64, T=64, T_out=32, packed=1, t=None, ks=1 << 14, vs=1 << 14, w=FARS[8], w_head=64, w_seq=256, seg=FAKE, keep_n=16, keep_dev=None,
          first=0, recent=0, kos=1 << 14, vos=1 << 14, wo=FARS[9], wo_head=32, wo_seq=128, keep=FARS[10], keep_head=32, keep_seq=128, seg_out=FARS[11]):
    t = {**{i: heads(FAR[i]) for i in range(4)}, **(t or {})}            # k, v, their outputs
    return B.lib().skipffn_kv_evict(n, H, D, T, T_out, packed, t[0], t[1], ks, vs, w, w_head, w_seq, seg, keep_n, keep_dev, first, recent, t[2], t[3],
                                    kos, vos, wo, wo_head, wo_seq, keep, keep_head, keep_seq, seg_out, None)


@pytest.mark.parametrize("packed", [0, 1])
def test_evict_rejects_bad_arguments(packed):
    for bad in (dict(n=-1), dict(H=0), dict(D=0), dict(T=-1), dict(T_out=-1), dict(first=-1), dict(recent=-1), dict(keep_n=-1), dict(seg=None),
                dict(seg=ODD), dict(seg_out=None), dict(keep_dev=ODD), dict(w=None), dict(w=FARS[8] + 2), dict(keep=None), dict(keep=FARS[10] + 1),
                dict(wo=FARS[9] + 2), dict(w_head=-1), dict(wo_head=31), dict(keep_head=31), dict(wo=FARS[8]), dict(t={3: heads(FAR[2])})):
        assert evict(packed=packed, **bad) == B.EINVAL, bad
    for bad in (dict(D=60), dict(D=136), dict(n=65536), dict(H=65536), dict(T=1 << 30), dict(T_out=1 << 30), dict(w_head=1 << 44)):
        assert evict(packed=packed, **bad) == B.ESHAPE, bad
    for i in range(4):
        assert evict(packed=packed, t={i: None}) == B.EINVAL and evict(packed=packed, t={i: heads(None)}) == B.EINVAL
        assert evict(packed=packed, t={i: heads(FAR[i], token=260)}) == B.ESHAPE
    for o in (2, 3):
        assert evict(packed=packed, t={o: heads(FAR[o], token=128)}) == B.EINVAL
        for i in (0, 1):
            assert evict(packed=packed, t={o: heads(FAR[i] + 1024)}) == B.EINVAL       # in place kept rows would race
    assert evict(packed=packed, n=0, seg=None) == B.OK


@pytest.mark.parametrize("packed", [0, 1])
def test_evict_rejects_counts_and_numbers_over_what_it_reads(packed):
    # a head's workgroup would write them while another's still reads
    for bad in (dict(seg_out=FAKE), dict(seg_out=FAKE + 4), dict(seg=FARS[11]), dict(keep_dev=FARS[11]), dict(keep_dev=FARS[11] + 4), dict(seg_out=FARS[8]),
                dict(keep=FARS[8]), dict(keep=FARS[8] + 64), dict(keep=FAKE), dict(keep=FARS[11]), dict(keep_dev=FARS[10]), dict(keep=FARS[9]),
                dict(wo=FAKE), dict(wo=FARS[11]), dict(wo=FARS[5], keep_dev=FARS[5])):
        assert evict(packed=packed, **bad) == B.EINVAL, bad


@pytest.mark.parametrize("packed", [0, 1])
def test_evict_rejects_numbers_weights_and_counts_over_the_rows(packed):
    # the second kernel copies rows by the numbers and offsets that the first one wrote
    last = 64 * 4 * 64 * 2 - 4                           # of a packed cache's keys, in bytes
    for i in range(4):                                   # k, v, their outputs
        for off in (0, 512, last if i < 2 else last // 2):
            for name in ("keep", "wo", "seg_out") + (("seg",) if i >= 2 else ()):
                assert evict(packed=packed, t={i: heads(FARS[12])}, **{name: FARS[12] + off}) == B.EINVAL, (i, off, name)
    for off in (4, 64, -64):                             # a head's numbers over the weights of another
        assert evict(packed=packed, wo=FARS[10] + off) == B.EINVAL, off


def test_evict_takes_outputs_side_by_side():
    """What counts is whether they share an element, not whether what they span meets.  n H 4 = 2^24 workgroups: more than a launch has, the last of
    the checks, so that nothing is enqueued."""
    n, H, T, D = 256, 1 << 14, 8, 8
    k = H * T * D                                        # elements of a sequence's keys
    w = H * T                                            # of its weights
    slab = 4 * k + 4 * w                                 # of 2 bytes: k, v, k_out, v_out, then weights_out and keep of 4 bytes
    t = {i: heads(FARS[12] + i * k * 2, token=D, head=T * D, H=H) for i in range(4)}
    far = {i: heads(FARS[4 + i], token=D, head=T * D, H=H) for i in range(4)}

    def call(wo, keep, head, seq, t=far, rows=k):
        return evict(n, H, D, T, T, 0, t, rows, rows, FARS[8], T, w, wo=wo, wo_head=head, wo_seq=seq, keep=keep, keep_head=head, keep_seq=seq, kos=rows,
                     vos=rows)
    assert call(FARS[9], FARS[10], T, w) == B.ESHAPE                     # accepted
    # weights and numbers of a head side by side; one of them a row on
    assert call(FARS[9], FARS[9] + 4 * T, 2 * T, 2 * w) == B.ESHAPE and call(FARS[9], FARS[9] + 4 * w, T, 2 * w) == B.ESHAPE
    assert call(FARS[9], FARS[9] + 4 * T - 4, 2 * T, 2 * w) == B.EINVAL and call(FARS[9], FARS[9] + 4 * w + 4, T, 2 * w) == B.EINVAL
    # all of a sequence in one place
    free = FARS[12] + 4 * k * 2
    out = {0: far[0], 1: far[1], 2: t[2], 3: t[3]}
    assert call(free, free + 4 * w, T, slab // 2, out, slab) == B.ESHAPE
    assert call(free - 4, free + 4 * w, T, slab // 2, out, slab) == B.EINVAL and call(free, free + 4 * w + 4, T, slab // 2, {**out, 2: t[0]}, slab) == B.EINVAL


def test_key_weights_reject_weights_over_the_saved_sums():
    assert key_weights(w=FARS[9], saved=FARS[9]) == B.EINVAL and key_weights(w=FARS[9] + 64, saved=FARS[9]) == B.EINVAL


def test_evict_rejects_sequences_that_lie_over_one_another():
    for bad in (dict(kos=64), dict(vos=1 << 12), dict(wo_seq=127), dict(keep_seq=127), dict(ks=-8), dict(wo_seq=-1),
                dict(t={2: heads(FAR[0] + (1 << 15) + 1024)})):          # the second sequence's keys
        assert evict(packed=0, **bad) == B.EINVAL, bad
    for bad in (dict(ks=4), dict(vos=12), dict(kos=1 << 44)):
        assert evict(packed=0, **bad) == B.ESHAPE, bad


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    bf = dict(dtype=torch.bfloat16)
    q, k = torch.zeros(8, 4, 64, **bf), torch.zeros(8, 2, 64, **bf)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    f, w, seg = torch.zeros(32), torch.zeros(2, 8), i32(2)
    for call in (lambda: B.skipffn_qk_rope_forward(q, k, q, k, i32(8), f), lambda: B.skipffn_qk_rope_backward(q, k, q, k, i32(8), f),
                 lambda: B.skipffn_attn_key_weights(q, k, seg, None, None, w), lambda: B.skipffn_kv_evict(k, k, w, seg, 4, k, k, w, i32(2, 8), seg),
                 lambda: B.skipffn_attn_decode_weights(q, k, k, seg, seg, None, None, None, q, w, None)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    for t in (torch.zeros(2, 8, dtype=torch.float64), torch.zeros(8, 2), torch.zeros(2, 16)[:, ::2]):
        with pytest.raises(ValueError, match="float32"):
            B._weights(t, (2, 8), "call", -1)
    assert B._weights(torch.zeros(2, 9)[:, :8], (2, 8), "call", -1)[1] == 9
    for t in (torch.zeros(31), torch.zeros(32, dtype=torch.float64), torch.zeros(64)[::2]):
        with pytest.raises(ValueError, match="float32"):
            B._floats(t, 32, "call", -1)
    for t in (torch.zeros(64), torch.zeros(63, **bf), torch.zeros(128, **bf)[::2]):
        with pytest.raises(ValueError, match="bfloat16"):
            B._gain(t, 64, "call", -1)
    with pytest.raises(ValueError, match="frequencies"):
        B._rope("call", -1, 8, i32(3, 8), f, [0] * 31)
    with pytest.raises(ValueError, match="int32"):
        B._rope("call", -1, 8, i32(3, 7), f, None)
