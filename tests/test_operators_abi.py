"""Refusals of the norm / rotation and packed attention entry points, on the host before any device call (CPU)."""

import ctypes

import numpy as np
import pytest
import torch

from paper_2606_25040_amd import ops

FAKE = 0x10000           # aligned, never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    return ops.load_library()


def t(ss=4 * 128, sh=128, data=FAKE, sb=0):
    return ops.Tensor(data, sb, ss, sh)


def by(x):
    return None if x is None else ctypes.byref(x)


def rotary(pairs=(22, 21, 21), adjacent=1, freq=1.0, n=None):
    return ops.Rotary(len(pairs) if n is None else n, (ctypes.c_int32 * 4)(*pairs), adjacent, (ctypes.c_double * 64)(*[freq] * 64))


def rope(lib, shape=(1, 10, 4, 128), Hk=4, q=None, k=..., norm=1, qw=FAKE, kw=FAKE, eps=1e-6, rot=..., pos=FAKE, pa=10, pb=0,
         qo=None, ko=..., dtype=ops.BF16):
    big = t(data=0x1000000)
    k = t(data=0x2000000) if k is ... else k
    ko = t(data=0x3000000) if ko is ... else ko
    rot = rotary() if rot is ... else rot
    return lib.chorus_qk_norm_rope(dtype, by(ops.Shape(*shape)), Hk, by(q or t()), by(k), norm, qw, kw, eps, by(rot), pos, pa, pb,
                                   by(qo or big), by(ko), None)


def test_norm_rope_refusals(lib):
    assert rope(lib, shape=(1, 10, 4, 64)) == 2
    assert rope(lib, shape=(0, 10, 4, 128)) == 1
    assert rope(lib, dtype=ops.FP8_E4M3) == 2
    assert rope(lib, k=None) == 1                                    # k_out and kv_heads without k
    assert rope(lib, ko=None) == 1
    assert rope(lib, Hk=0) == 1
    assert rope(lib, norm=3) == 1
    assert rope(lib, qw=None) == 1
    assert rope(lib, kw=None) == 1
    assert rope(lib, norm=0) == 1                                    # weights without a norm
    assert rope(lib, qw=FAKE + 4) == 1
    assert rope(lib, eps=-1.0) == 1 and rope(lib, eps=float("nan")) == 1
    assert rope(lib, norm=2, shape=(1, 10, 129, 128)) == 2
    assert rope(lib, norm=2, Hk=129) == 2
    assert rope(lib, norm=0, qw=None, kw=None, rot=None, pos=None) == 1
    assert rope(lib, rot=None) == 1 and rope(lib, pos=None) == 1
    assert rope(lib, rot=rotary(n=0)) == 1 and rope(lib, rot=rotary(n=5)) == 1
    assert rope(lib, rot=rotary((22, 21, 20))) == 1
    assert rope(lib, rot=rotary((70, -6))) == 1
    assert rope(lib, rot=rotary(adjacent=2)) == 1
    assert rope(lib, rot=rotary(freq=float("inf"))) == 1
    assert rope(lib, pa=-1) == 1 and rope(lib, pb=-1) == 1
    assert rope(lib, pos=FAKE + 2) == 1
    assert rope(lib, shape=(1 << 14, 1 << 14, 64, 128)) == 2
    assert rope(lib, q=t(data=FAKE + 8)) == 1
    assert rope(lib, q=t(ss=4 * 128 + 4)) == 1
    assert rope(lib, qo=t(data=FAKE + 512)) == 1                     # overlaps its input, shifted
    assert b"overlap" in lib.chorus_last_error()
    assert rope(lib, qo=t(ss=8 * 128)) == 1                          # or with other strides
    assert rope(lib, qo=t(data=0x2000000)) == 1 and rope(lib, ko=t()) == 1 and rope(lib, ko=t(data=0x1000000)) == 1


def test_norm_rope_refuses_more_heads_than_a_launch_holds(lib):
    far = dict(qo=t(data=1 << 40), ko=t(data=1 << 44))
    assert rope(lib, shape=(1, 1, (1 << 22) + 1, 128), **far) == 2
    assert rope(lib, shape=(1, 1, 4, 128), Hk=(1 << 22) + 1, k=t(data=1 << 46), **far) == 2


def test_norm_rope_of_no_tokens(lib):
    null = t(data=None)
    assert rope(lib, shape=(2, 0, 4, 128), q=null, k=null, qo=null, ko=null) == 0
    assert rope(lib, shape=(2, 0, 4, 64)) == 2 and rope(lib, shape=(2, -1, 4, 128)) == 1 and rope(lib, shape=(0, 0, 4, 128)) == 1
    assert rope(lib, shape=(2, 0, 4, 128), dtype=ops.FP8_E4M3) == 2


def packed(n=2, tq=10, tk=20, prefix=0, H=4, Hk=2, D=128, causal=1, max_q=0):
    return ops.PackedShape(n, tq, tk, prefix, H, Hk, D, causal, max_q)


BAD = [(packed(n=0), 1), (packed(tq=-1), 1), (packed(tk=-1), 1), (packed(prefix=-1), 1), (packed(max_q=-1), 1), (packed(H=5), 1),
       (packed(Hk=0), 1), (packed(H=0, Hk=1), 1), (packed(D=64), 2), (packed(causal=2), 1), (packed(n=(1 << 20) + 1), 2),
       (packed(tq=1 << 30), 2), (packed(H=70000, Hk=70000, tq=1), 2), (packed(tk=(1 << 30) + 1), 2),
       (packed(prefix=(1 << 30) + 1), 2), (packed(tq=1 << 27, H=8, Hk=8, n=1 << 20), 2)]


def make_plan(lib, s, qo=FAKE, ko=FAKE, kl=None, plan=FAKE, nbytes=None):
    need = lib.chorus_packed_plan_bytes(by(s)) if nbytes is None else nbytes
    return lib.chorus_plan_packed_attn(by(s), qo, ko, kl, plan, need, None)


def attend(lib, s, q=None, k=..., v=..., pk=None, pv=None, sm=0.088, plan=FAKE, nbytes=None, out=None, ws=FAKE, ws_bytes=None,
           dtype=ops.F16):
    need = lib.chorus_packed_plan_bytes(by(s)) if nbytes is None else nbytes
    wsb = lib.chorus_packed_attn_workspace_size(by(s)) if ws_bytes is None else ws_bytes
    k = t() if k is ... else k
    v = t() if v is ... else v
    return lib.chorus_packed_attn_fwd(dtype, by(s), by(q or t()), by(k), by(v), by(pk), by(pv), sm, plan, need, by(out or t(data=0x9000000)), None,
                                      ws, wsb, None)


def test_packed_shapes_are_checked_everywhere(lib):
    for s, status in BAD:
        assert lib.chorus_packed_plan_bytes(by(s)) == 0 and lib.chorus_packed_attn_workspace_size(by(s)) == 0
        assert make_plan(lib, s) == status
        assert attend(lib, s) == status
    assert lib.chorus_packed_plan_bytes(None) == 0
    assert lib.chorus_packed_plan_bytes(by(packed())) > 0


def test_packed_plan_refusals(lib):
    s = packed()
    assert make_plan(lib, s, qo=None) == 1 and make_plan(lib, s, ko=None) == 1
    assert make_plan(lib, s, kl=FAKE + 2) == 1
    assert make_plan(lib, s, plan=None) == 1 and make_plan(lib, s, plan=FAKE + 16) == 1
    assert make_plan(lib, s, nbytes=256) == 3


def test_packed_attention_refusals(lib):
    s = packed()
    assert attend(lib, s, dtype=ops.FP8_E4M3) == 2
    assert attend(lib, s, q=t(data=FAKE + 2)) == 1
    assert attend(lib, s, k=None) == 1 and attend(lib, s, v=None) == 1
    assert attend(lib, s, k=t(ss=1 << 30)) == 2
    assert attend(lib, s, out=t(ss=-128)) == 1
    assert attend(lib, s, out=t()) == 1                              # k's memory
    assert attend(lib, s, pk=t(), pv=t()) == 1                       # a prefix that the shape does not have
    assert attend(lib, packed(prefix=5)) == 1                        # and one that is missing
    assert attend(lib, packed(prefix=5), pk=t()) == 1
    assert attend(lib, s, sm=0.0) == 1 and attend(lib, s, sm=float("inf")) == 1
    assert attend(lib, s, plan=None) == 1 and attend(lib, s, plan=FAKE + 64) == 1
    assert attend(lib, s, nbytes=512) == 3
    assert attend(lib, s, ws=None) == 5 and attend(lib, s, ws_bytes=256) == 5
    assert attend(lib, packed(tq=0), q=t(data=None)) == 0            # nothing to do


def test_python_refuses_host_tensors():
    x = torch.zeros(1, 4, 2, 128, dtype=torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        ops.qk_norm_rope(x, norm="head", q_weight=torch.ones(128))
    o = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        ops.plan_packed_attn(o, o, 1, 1, 1, 1)
    with pytest.raises(ValueError, match="norm must be"):
        ops.qk_norm_rope(x, norm="batch")
    for bad in ((64, 1), (), (10,) * 5, (65, -1)):
        with pytest.raises(ValueError, match="pairs"):
            ops.RotaryAxes(bad)
    with pytest.raises(ValueError, match="freqs"):
        ops.RotaryAxes((64,), freqs=[1.0] * 63)


ROW = 2 * 128            # bytes of one head of one token


def test_packed_outputs_that_share_memory_are_refused(lib):
    """Told by the workspace check behind: 5 is a call that passed, and nothing is launched either way."""
    s = packed(tq=10, tk=20, prefix=6, H=4, Hk=2)
    far = dict(k=t(data=0x2000000), v=t(data=0x3000000), pk=t(data=0x4000000), pv=t(data=0x5000000), ws=None)
    base = 0x100000

    def status(q=None, out=None, **kw):
        st = attend(lib, s, q=q or t(data=base), out=out or t(data=0x9000000), **(far | kw))
        if st == 1:
            assert b"overlaps" in lib.chorus_last_error()
        return st

    assert status() == 5 and status(out=t(data=base)) == 5                   # apart; in place
    assert status(out=t(128, 4 * 128, base)) == 1                            # q transposed, at the same address
    assert status(q=t(4 * 128, 128, base), out=t(4 * 128, 128, base + ROW)) == 1
    for shift, st in ((1, 1), (4, 1), (39, 1), (-39, 1), (40, 5), (-40, 5)):   # moved by heads within one buffer
        assert status(out=t(data=base + shift * ROW)) == st
    # views of one fused row of 12 heads: q 0 - 3, k 4 - 5, v 6 - 7, out from 8 or from inside another
    f = dict(q=t(12 * 128, 128, base), k=t(12 * 128, 128, base + 4 * ROW), v=t(12 * 128, 128, base + 6 * ROW))
    for head, st in ((0, 5), (1, 1), (3, 1), (4, 1), (5, 1), (7, 1), (8, 5), (9, 1), (11, 1)):
        assert status(out=t(12 * 128, 128, base + head * ROW), **f) == st, head
    assert status(out=t(12 * 128, 128, base + 12 * 20 * ROW), **f) == 5       # behind all rows
    # head-major: [heads, rows, 128] buffers of 20 rows a head, k in heads 4 - 5 of it
    m = dict(q=t(128, 20 * 128, base), k=t(128, 20 * 128, base + 80 * ROW))
    for row, st in ((0, 5), (5, 1), (10, 5), (75, 1), (80, 1), (120, 5)):
        assert status(out=t(128, 20 * 128, base + row * ROW), **m) == st, row
    for name in ("k", "v", "pk", "pv"):
        rows = 6 if name[0] == "p" else 20
        last = (rows - 1) * 4 * 128 * 2 + ROW
        assert status(out=t(data=far[name].data + last)) == 1                # in its last row's second head
        assert status(out=t(data=far[name].data + last + ROW)) == 5
    # one token and one head: strides that reach nowhere
    s = packed(tq=1, tk=1, prefix=1, H=1, Hk=1)
    assert status(q=t(7 * 128, 5 * 128, base), out=t(128, 128, base)) == 5


def test_norm_rope_outputs_that_share_memory_are_refused(lib):
    base = 0x100000

    def refused(qo, ko, q=t(12 * 128, 128, base, 99 * 12 * 128), k=t(12 * 128, 128, base + 4 * ROW, 99 * 12 * 128)):
        st = rope(lib, shape=(3, 10, 4, 128), Hk=2, q=q, k=k, qo=qo, ko=ko)
        return st == 1 and b"overlaps" in lib.chorus_last_error()

    def view(head, token=0, request=0):
        return t(12 * 128, 128, base + (head + 12 * token + 12 * 99 * request) * ROW, 99 * 12 * 128)

    far = t(data=0x9000000, sb=10 * 512)
    assert refused(view(1), far) and refused(view(0, 1), far)          # q's own memory, shifted
    assert refused(view(4), far) and refused(view(2, 9, 2), far)       # k's
    assert refused(far, view(3)) and refused(far, view(5))             # q's and k's, from k_out
    assert refused(view(8), view(10)) and refused(view(8), view(11)) and refused(view(7), view(6, 3))   # each other's
    assert refused(t(128, 512, base, 99 * 12 * 128), far)              # at q's address, other strides
    # k in a buffer of its own; q_out shifted into it; k_out shifted into q_out
    k, out = t(2 * 128, 128, 0x700000, 10 * 2 * 128), t(4 * 128, 128, 0xA00000, 10 * 4 * 128)
    assert refused(t(4 * 128, 128, 0x700000 + ROW, 10 * 4 * 128), far, k=k)
    assert refused(out, t(4 * 128, 128, 0xA00000 + 3 * ROW, 10 * 4 * 128), k=k)
    assert refused(far, t(2 * 128, 128, base + 3 * ROW, 10 * 2 * 128), k=k)


def test_outputs_are_told_apart_as_by_their_bytes(lib):
    """Random places, counts and strides, of rows that overlap each other too: what passes shares no byte, and what shares
    none passes where the strides between tokens and between heads are the same."""
    def chunks(x, rows, heads):
        at = x.data // 16 + (np.arange(rows)[:, None] * x.stride_s + np.arange(heads) * x.stride_h).reshape(-1, 1) // 8
        return set((at + np.arange(16)).ravel().tolist())

    rng = np.random.default_rng(6)
    passed = exact = 0
    for _ in range(3000):
        tq, tk, H, Hk = (int(n) for n in rng.integers(1, 5, 4))
        alike = rng.random() < 0.6
        ss, sh = (8 * int(n) for n in rng.choice([0, 1, 15, 16, 17, 32, 48, 64, 80, 128, 160], 2))
        out = t(ss, sh, 0x100000)
        if not alike:
            ss, sh = (8 * int(n) for n in rng.choice([0, 1, 15, 16, 17, 32, 48, 64, 80, 128, 160], 2))
        k = t(ss, sh, 0x100000 + 16 * int(rng.integers(-300, 300)))
        st = attend(lib, packed(tq=tq, tk=tk, H=H * Hk, Hk=Hk), q=t(data=0x9000000), k=k, v=t(data=0x8000000), out=out, ws=None)
        assert st in (1, 5)
        shared = bool(chunks(out, tq, H * Hk) & chunks(k, tk, Hk))
        assert not (shared and st == 5), (tq, tk, H, Hk, out.data, out.stride_s, out.stride_h, k.data, k.stride_s, k.stride_h)
        passed += st == 5
        inner, outer = sorted((ss, sh))
        if alike and not shared and inner >= 128 and outer >= inner * max(H * Hk if inner == sh else tq, Hk if inner == sh else tk):
            exact += 1
            assert st == 5
    assert passed > 500 and exact > 100


def test_a_plan_needs_its_whole_buffer(lib):
    s = packed()
    need = lib.chorus_packed_plan_bytes(by(s))
    with pytest.raises(ValueError, match="shorter"):
        ops.PackedPlan(torch.zeros(need - 1, dtype=torch.uint8), s)
    data = torch.zeros(need + 256, dtype=torch.uint8)
    assert ops.PackedPlan(data, s).plan_bytes == need
    at = ops._aligned(data) - data.data_ptr()
    assert ops.PackedPlan(data[at:at + need], s).plan_bytes == need
    with pytest.raises(ValueError, match="shorter"):
        ops.PackedPlan(data[at + 16:at + 16 + need], s)


def test_ladder_of_each_axis():
    r = ops.RotaryAxes((2, 62), theta=100.0)
    assert r.freqs[:3] == (1.0, 100.0 ** -0.5, 1.0) and r.freqs[63] == 100.0 ** (-61 / 62)


def test_rows_that_share_memory_are_no_output():
    x = torch.zeros(6, 1, 128)
    ops._writable(x, "out")
    ops._writable(x.transpose(0, 1), "out")
    for bad in (x[:1].expand(6, 1, 128), torch.zeros(1000).as_strided((5, 2, 128), (128, 64, 1))):
        with pytest.raises(ValueError, match="share memory"):
            ops._writable(bad, "out")
