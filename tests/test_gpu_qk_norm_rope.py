"""Norm and rotation of Q and K against the float64 oracle, through the C ABI.

Tolerance: the one rounding of the output is half a step of its type (eps / 2 relative; f16 also half its smallest
step, 2^-25, near zero).  The fp32 arithmetic before it is some ten roundings of 2^-24 for the norm and an angle
within 2^-22 rad, on values no larger than the pair's length: 2^-19 of that length covers them."""

import numpy as np
import pytest
import torch

from oracle import rotary as orc
from paper_2606_25040_amd import ops

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    ops.load_library()
    torch.cuda.set_device(0)
    yield


F16, BF16 = torch.float16, torch.bfloat16


def draw(shape, dtype, seed, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def weight(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.3 * torch.randn(*shape, generator=g)).cuda()


def check(got, x, rot, positions, norm, w, eps):
    f = dict(positions=None) if rot is None else dict(positions=positions.cpu().numpy(), pairs=rot.pairs,
                                                      freqs=rot.freqs, adjacent=rot.adjacent)
    x = x.float().cpu().numpy()
    want = orc.norm_rotate(x, norm, None if w is None else w.cpu().numpy(), eps, **f)
    if rot is None:
        length = np.abs(want)
    else:
        y = orc.norm(x, norm, None if w is None else w.cpu().numpy(), eps)
        a, b = (y[..., 0::2], y[..., 1::2]) if rot.adjacent else (y[..., :64], y[..., 64:])
        r = np.hypot(a, b)
        length = np.repeat(r, 2, -1) if rot.adjacent else np.concatenate((r, r), -1)
    fi = torch.finfo(got.dtype)
    tol = fi.eps / 2 * np.abs(want) + 2.0 ** -19 * length + (2.0 ** -25 if got.dtype == F16 else 0)
    err = np.abs(got.float().cpu().numpy() - want)
    assert got.shape == want.shape
    assert (err <= tol).all(), f"worst {float((err - tol).max())} at {np.unravel_index((err - tol).argmax(), err.shape)}"


CASES = [  # B, S, H, Hk, dtype, norm, pairs, adjacent
    (1, 1, 1, 1, F16, "head", (64,), False),
    (2, 1, 32, 8, BF16, "head", (64,), True),
    (1, 37, 5, 5, BF16, "token", (22, 21, 21), True),
    (3, 19, 12, 3, F16, "none", (22, 21, 21), True),
    (2, 100, 7, 1, F16, "token", (16, 24, 24), False),
    (1, 300, 40, 40, BF16, "token", (22, 21, 21), True),
    (1, 9, 128, 3, BF16, "token", (32, 32), False),
    (1, 9, 200, 70, F16, "head", (0, 60, 4, 0), True),
    (2, 65, 24, 24, BF16, "head", (16, 24, 24), False),
    (1, 41, 3, 0, BF16, "head", (22, 21, 21), False),
    (2, 33, 6, 2, F16, "head", None, True),
    (1, 1111, 9, 2, BF16, "token", None, True),
    (1, 4999, 2, 1, F16, "none", (64,), False),
    (3, 7000, 1, 1, BF16, "token", (64,), True),       # workgroups that take several tokens, across requests
    (1, 2500, 64, 0, F16, "token", (32, 32), False),
]


@pytest.mark.parametrize("B,S,H,Hk,dtype,norm,pairs,adjacent", CASES)
def test_matches_the_oracle(B, S, H, Hk, dtype, norm, pairs, adjacent):
    norm = None if norm == "none" else norm
    q, k = draw((B, S, H, 128), dtype, 1), draw((B, S, Hk, 128), dtype, 2, 0.4) if Hk else None
    rot = pos = None
    if pairs:
        rot = ops.RotaryAxes(pairs, adjacent=adjacent)
        g = torch.Generator().manual_seed(3)
        pos = torch.randint(0, 5000, (len(pairs), B, S), generator=g, dtype=torch.int32).cuda()
    wq = wk = None
    if norm:
        wq = weight((128,) if norm == "head" else (H, 128), 4)
        wk = weight((128,) if norm == "head" else (Hk * 128,), 5) if Hk else None
    got = ops.qk_norm_rope(q, k, rotary=rot, positions=pos, norm=norm, q_weight=wq, k_weight=wk, eps=1e-5)
    torch.cuda.synchronize()
    check(got[0] if Hk else got, q, rot, pos, norm, wq, 1e-5)
    if Hk:
        check(got[1], k, rot, pos, norm, wk, 1e-5)


@pytest.mark.parametrize("adjacent", [True, False])
def test_far_and_negative_positions(adjacent):
    q = draw((1, 8, 2, 128), BF16, 7)
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 10 ** 9, -123456789]], dtype=torch.int32).cuda()
    rot = ops.RotaryAxes((64,), adjacent=adjacent)
    # the oracle's own float64 angle of 2^31 is off by up to 2^-22 rad, as the kernel's is: within 2^-19 of the length
    check(ops.qk_norm_rope(q, rotary=rot, positions=pos), q, rot, pos, None, None, 0.0)


def test_pairs_with_frequency_zero_do_not_turn():
    q = draw((1, 5, 3, 128), F16, 8)
    rot = ops.RotaryAxes((64,), freqs=[1.0] * 16 + [0.0] * 48, adjacent=False)
    got = ops.qk_norm_rope(q, rotary=rot, positions=torch.arange(5, dtype=torch.int32).cuda()[None])
    keep = torch.tensor([i % 64 >= 16 for i in range(128)]).cuda()
    assert torch.equal(got[..., keep], q[..., keep])
    assert not torch.equal(got[:, 1:][..., ~keep], q[:, 1:][..., ~keep])


@pytest.mark.parametrize("norm", ["head", "token", None])
def test_strided_views_shared_positions_and_in_place(norm):
    B, S, H, Hk = 2, 50, 6, 2
    fused = draw((B, S, (H + 2 * Hk), 128), BF16, 9)
    q, k = fused[:, :, :H], fused[:, :, H:H + Hk]
    rot = ops.RotaryAxes((22, 21, 21))
    pos = torch.randint(0, 40, (3, S), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).cuda()
    ws = {None: (None, None), "head": (weight((128,), 1), weight((128,), 2)),
          "token": (weight((H, 128), 1), weight((Hk, 128), 2))}[norm]
    kw = dict(rotary=rot, positions=pos, norm=norm, q_weight=ws[0], k_weight=ws[1])
    out = torch.empty(B, H, S, 128, dtype=BF16, device="cuda").transpose(1, 2)
    want = ops.qk_norm_rope(q, k, q_out=out, **kw)
    check(want[0], q, rot, pos, norm, ws[0], 1e-6)
    check(want[1], k, rot, pos, norm, ws[1], 1e-6)
    plain = ops.qk_norm_rope(q.contiguous(), k.contiguous(), **kw)
    assert torch.equal(plain[0], want[0]) and torch.equal(plain[1], want[1])
    rest = fused[:, :, H + Hk:].clone()
    got = ops.qk_norm_rope(q, k, q_out=q, k_out=k, **kw)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, :, H + Hk:], rest)


@pytest.mark.parametrize("heads_first", [False, True])
def test_outputs_between_the_inputs_of_one_buffer(heads_first):
    B, S, H, Hk = 2, 21, 4, 2
    rot, pos = ops.RotaryAxes((64,)), torch.arange(S, dtype=torch.int32).cuda()[None]
    shape = (B, 2 * (H + Hk), S, 128) if heads_first else (B, S, 2 * (H + Hk), 128)
    buf = draw(shape, BF16, 21)
    rows = buf.transpose(1, 2) if heads_first else buf
    q, qo, k, ko = rows.split((H, H, Hk, Hk), 2)
    was = buf.clone().transpose(1, 2) if heads_first else buf.clone()
    want = ops.qk_norm_rope(q, k, rotary=rot, positions=pos)
    ops.qk_norm_rope(q, k, rotary=rot, positions=pos, q_out=qo, k_out=ko)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    assert torch.equal(q, was[:, :, :H]) and torch.equal(k, was[:, :, 2 * H:2 * H + Hk])


@pytest.mark.parametrize("norm", ["head", "token", None])
def test_a_token_or_head_that_is_not_finite_stays_alone(norm):
    q = draw((1, 20, 8, 128), F16, 10)
    bad = q.clone()
    bad[0, 3, 2, 5], bad[0, 11, 0, 77] = float("nan"), float("inf")
    w = None if norm is None else weight((128,) if norm == "head" else (8, 128), 3)
    rot, pos = ops.RotaryAxes((64,)), torch.arange(20, dtype=torch.int32).cuda()[None]
    kw = dict(rotary=rot, positions=pos, norm=norm, q_weight=w)
    a, b = ops.qk_norm_rope(q, **kw), ops.qk_norm_rope(bad, **kw)
    hit = torch.zeros(1, 20, 8, dtype=torch.bool)
    hit[0, 3, :, ], hit[0, 11, :] = norm == "token", norm == "token"
    hit[0, 3, 2] = hit[0, 11, 0] = True
    hit = hit.cuda()
    assert torch.equal(a[~hit], b[~hit])
    assert torch.isnan(b[0, 3, 2]).any() and not torch.isfinite(b[0, 11, 0]).all()


@pytest.mark.parametrize("norm,H", [("head", 3), ("token", 40), ("token", 128), ("token", 1)])
def test_norm_of_values_whose_squares_leave_the_range(norm, H):
    """Of bf16 values around 2^-115 to 2^122; an ordinary token between them, and eps of the size of the mean."""
    scales = [120, 64, 61, 58, 55, 0, -40, -52, -60, -75, -80, -115]
    every = draw((1, len(scales), H, 128), BF16, 13)
    for s, e in enumerate(scales):
        every[0, s] *= 2.0 ** e
    w = weight((128,) if norm == "head" else (H, 128), 14)
    for eps, rows in ((2.0 ** 120, 6), (2.0 ** -120, 12), (1e-6, 12), (0.0, 12)):   # (results stay above 2^-126)
        q = every[:, :rows].contiguous()
        kw = dict(norm=norm, q_weight=w, eps=eps)
        check(ops.qk_norm_rope(q, **kw), q, None, None, norm, w, float(np.float32(eps)))
        both = ops.qk_norm_rope(q, q[:, :, :1].clone(), k_weight=w if norm == "head" else w[:1].contiguous(), **kw)
        assert torch.equal(both[0], ops.qk_norm_rope(q, **kw))
    rot, pos = ops.RotaryAxes((64,)), torch.arange(len(scales), dtype=torch.int32).cuda()[None]
    check(ops.qk_norm_rope(q, rotary=rot, positions=pos, norm=norm, q_weight=w, eps=0.0), q, rot, pos, norm, w, 0.0)


def test_no_tokens():
    """As packed attention takes a batch without queries."""
    q, k = (torch.empty(1, 0, h, 128, dtype=BF16, device="cuda") for h in (4, 2))
    rot, pos = ops.RotaryAxes((22, 21, 21)), torch.empty(3, 0, dtype=torch.int32, device="cuda")
    got = ops.qk_norm_rope(q, k, rotary=rot, positions=pos, norm="head", q_weight=weight((128,), 1), k_weight=weight((128,), 2))
    assert got[0].shape == q.shape and got[1].shape == k.shape
    assert ops.qk_norm_rope(q, rotary=rot, positions=pos, q_out=q) is q


def test_zero_rows_give_zero():
    q = torch.zeros(1, 3, 2, 128, dtype=BF16, device="cuda")
    assert not ops.qk_norm_rope(q, norm="head", q_weight=weight((128,), 1)).any()


def test_captured_and_on_another_stream():
    q, k = draw((1, 500, 4, 128), BF16, 11), draw((1, 500, 4, 128), BF16, 12)
    rot, pos = ops.RotaryAxes((22, 21, 21)), torch.randint(0, 99, (3, 500), dtype=torch.int32).cuda()
    kw = dict(rotary=rot, positions=pos, norm="head", q_weight=weight((128,), 1), k_weight=weight((128,), 2))
    want = ops.qk_norm_rope(q, k, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = ops.qk_norm_rope(q, k, **kw)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    outs = [torch.empty_like(q), torch.empty_like(k)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.qk_norm_rope(q, k, q_out=outs[0], k_out=outs[1], **kw)
    for shift in (0, 5, 11):
        pos.add_(shift)
        want = ops.qk_norm_rope(q, k, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_refusals_of_the_binding():
    q, k, w = draw((2, 5, 4, 128), BF16, 1), draw((2, 5, 2, 128), BF16, 2), weight((128,), 3)
    rot, pos = ops.RotaryAxes((32, 32)), torch.zeros(2, 5, dtype=torch.int32, device="cuda")

    def no(match, kind=ValueError, **kw):
        with pytest.raises(kind, match=match):
            ops.qk_norm_rope(**(dict(q=q, k=k) | kw))

    no("go together", rotary=rot)
    no("positions must be", rotary=rot, positions=pos.long())
    no("positions must be", rotary=rot, positions=pos[:1])
    no("positions must be", rotary=rot, positions=pos[:, :4])
    no("k must share", k=k[:, :4], rotary=rot, positions=pos)
    no("k must share", k=k.to(F16), rotary=rot, positions=pos)
    no("a weight must be", norm="token", q_weight=w, k_weight=w)
    no("a weight must be", q_weight=w, rotary=rot, positions=pos)
    no("a weight is given", RuntimeError, norm="head", q_weight=w)
    no("neither", RuntimeError)
    no("q_out must have", rotary=rot, positions=pos, q_out=q[:1])
    no("share memory", rotary=rot, positions=pos, q_out=q[:1].expand(2, 5, 4, 128))
    no("overlaps", RuntimeError, rotary=rot, positions=pos, k=q, k_out=q.clone(), q_out=q)
    no("k_out without k", k=None, k_out=k, rotary=rot, positions=pos)
