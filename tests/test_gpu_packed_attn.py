"""Attention over packed sequences against the float64 oracle, through the C ABI.

Tolerance of an output, with W = sum_c p_c |v_c| (the oracle on |V|) and A = the row's largest sm_scale sum_d |q_d k_d|:
the stored value is off by half a step of its type (eps / 2 relative, f16 also 2^-25); every weight is rounded to that
type for the second product, eps / 2 of W; a score is a sum of 128 products, off by 132 x 2^-24 A, and one rounding of
2^-23 (A + 16) more in the exponent's argument, which moves a weight by that much relative to 1, twice (itself and the
sum); fp32 sums of n weights add n 2^-25.  lse: the score's error and the sum's, and 2^-22 of its own size."""

import numpy as np
import pytest
import torch

from oracle import packed as orc
from paper_2606_25040_amd import ops

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
SM = 128 ** -0.5


@pytest.fixture(scope="module", autouse=True)
def device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    ops.load_library()
    torch.cuda.set_device(0)
    yield


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def offsets(n):
    return [0] + [int(x) for x in np.cumsum(n)]


class Batch:
    """Sequences of nq queries and nk keys, packed; `cache`: keys in rows of their own with NaN behind them."""

    def __init__(self, nq, nk, H, Hk, dtype, causal=True, prefix=0, cache=False, seed=0, scale=1.5):
        g = torch.Generator().manual_seed(seed)

        def draw(*shape, s=1.0):
            return (torch.randn(*shape, generator=g) * s).to(dtype).cuda()

        self.nq, self.nk, self.causal = list(nq), list(nk), causal
        self.qo = offsets(nq)
        room = max(nk) + 7
        self.ko = [room * i for i in range(len(nk) + 1)] if cache else offsets(nk)
        self.cache = cache
        self.q = draw(self.qo[-1], H, 128, s=scale)
        self.k, self.v = draw(self.ko[-1], Hk, 128), draw(self.ko[-1], Hk, 128)
        if cache:
            for i, n in enumerate(nk):
                self.k[self.ko[i] + n:self.ko[i + 1]] = float("nan")
                self.v[self.ko[i] + n:self.ko[i + 1]] = float("nan")
        self.pk = self.pv = None
        if prefix:
            self.pk, self.pv = draw(prefix, Hk, 128), draw(prefix, Hk, 128)

    def plan(self, max_q=None, out=None):
        return ops.plan_packed_attn(ints(self.qo), ints(self.ko), self.q.shape[0], self.k.shape[0], self.q.shape[1],
                                    self.k.shape[1], causal=self.causal, k_lens=ints(self.nk) if self.cache else None,
                                    prefix=0 if self.pk is None else self.pk.shape[0],
                                    max_q=max(self.nq) if max_q is None else max_q, out=out)

    def run(self, plan=None, **kw):
        got = ops.packed_attn_fwd(self.q, self.k, self.v, plan or self.plan(), prefix_k=self.pk, prefix_v=self.pv,
                                  return_lse=True, **kw)
        torch.cuda.synchronize()
        return got

    def oracle(self, absolute=False, sm=SM):
        q, k, v, pk, pv = (None if x is None else x.float().cpu().numpy() for x in (self.q, self.k, self.v, self.pk, self.pv))
        if absolute:
            v, pv = np.abs(v), None if pv is None else np.abs(pv)
        return orc.attention(q, k, v, self.qo, self.ko, sm, self.causal, self.nk if self.cache else None, pk, pv)

    def check(self, got, sm=SM):
        O, lse = self.oracle(sm=sm)
        W, _ = self.oracle(absolute=True, sm=sm)
        kk = self.k.float().cpu().numpy()
        largest = np.abs(kk[np.isfinite(kk)]).max() if kk.size else 0.0
        if self.pk is not None:
            largest = max(largest, float(self.pk.float().abs().max()))
        A = sm * np.abs(self.q.float().cpu().numpy()).sum(-1) * largest                     # [total_q, H], above the true one
        n = max(self.nk) + (0 if self.pk is None else self.pk.shape[0])
        ds = 132 * 2.0 ** -24 * A + 2.0 ** -23 * (A + 16)
        fi = torch.finfo(self.q.dtype)
        tol = fi.eps / 2 * np.abs(O) + (fi.eps / 2 + 2 * ds[..., None] + n * 2.0 ** -25) * W
        tol += 2.0 ** -25 if self.q.dtype == F16 else 0
        out, l = got[0].float().cpu().numpy(), got[1].cpu().numpy()
        err = np.abs(out - O)
        assert (err <= tol).all(), f"worst {float((err - tol).max())} at {np.unravel_index((err - tol).argmax(), err.shape)}"
        none = np.isneginf(lse)
        assert np.array_equal(np.isneginf(l), none) and not out.transpose(1, 0, 2)[none].any()
        tl = ds.T + n * 2.0 ** -25 + 2.0 ** -22 * (1 + np.abs(np.where(none, 0, lse)))
        assert (np.abs(l[~none] - lse[~none]) <= tl[~none]).all()


def near(got, clean, W, rows):
    """Equal but for rounding: when one row of a wave moves its running maximum, the others' weights are rounded
    relative to other maxima (eps / 2 of W on each side, and eps / 2 of the value; fp32 parts below 1e-4 here)."""
    eps = torch.finfo(got[0].dtype).eps
    a, c = (x[0][rows].float().cpu().numpy() for x in (got, clean))
    assert (np.abs(a - c) <= eps * np.abs(c) + (eps + 1e-4) * W[rows] + 2.0 ** -24).all()
    assert float((got[1][:, rows] - clean[1][:, rows]).abs().max()) <= 1e-4


CASES = {  # nq, nk, H, Hk, dtype, causal, prefix, cache
    "one_token_one_key": ([1], [1], 1, 1, F16, True, 0, False),
    "tokens_of_short_caches": ([1] * 4, [1, 63, 64, 300], 8, 2, BF16, True, 0, True),
    "token_of_a_long_cache": ([1], [5000], 5, 1, F16, True, 0, False),
    "tokens_full_heads": ([1, 1, 1], [700, 65, 1], 12, 12, BF16, True, 0, True),
    "drafts": ([4, 1, 3, 4], [1024, 1, 129, 90], 10, 2, F16, True, 0, True),
    "edges_causal": ([1, 31, 32, 33, 63, 64, 65, 127, 128, 129], [1, 31, 32, 33, 63, 64, 65, 127, 128, 129], 2, 2, BF16, True,
                     0, False),
    "edges_full": ([1, 31, 33, 64, 65, 129], [129, 1, 64, 65, 127, 2], 3, 1, F16, False, 0, False),
    "empty_sequences": ([0, 5, 0, 7, 0], [4, 0, 0, 9, 3], 4, 4, BF16, False, 0, False),
    "empty_sequences_causal": ([0, 5, 0, 7, 0, 2], [4, 0, 0, 9, 3, 1], 4, 2, F16, True, 0, False),
    "more_queries_than_keys": ([70, 300, 5], [10, 129, 0], 2, 1, BF16, True, 0, False),
    "context_ahead": ([17, 100, 1], [217, 164, 900], 6, 2, F16, True, 0, False),
    "group_of_five": ([77, 40], [77, 40], 5, 1, BF16, True, 0, False),
    "group_of_three": ([200, 1, 50], [200, 64, 50], 9, 3, F16, True, 0, True),
    "long_causal": ([1500], [1500], 2, 1, BF16, True, 0, False),
    "long_full": ([333, 1200], [333, 1200], 1, 1, F16, False, 0, False),
    "heads_beyond_eight": ([150], [150], 11, 11, BF16, True, 0, False),
    "group_of_forty": ([1, 9, 0, 33], [200, 9, 5, 70], 40, 1, BF16, True, 0, True),
    "prefix_group_of_forty": ([1, 2, 1, 1], [3, 70, 1, 200], 40, 1, F16, True, 130, True),
    "prefix_of_one": ([1, 2], [1, 5], 4, 2, BF16, True, 1, False),
    "prefix_tokens": ([1] * 40, list(range(1, 41)), 8, 2, F16, True, 1000, True),
    "prefix_tokens_exact_blocks": ([1] * 9, [64] * 9, 4, 4, BF16, True, 128, False),
    "prefix_without_own_keys": ([1, 3, 2], [0, 0, 1], 3, 1, F16, True, 65, False),
    "prefix_prompts": ([130, 257, 20], [130, 300, 20], 4, 2, BF16, True, 333, False),
    "prefix_half_tiles": ([16, 15, 1, 30], [16, 15, 60, 30], 8, 2, BF16, True, 500, False),
    "prefix_pooled_and_cut": ([1, 2, 1], [900, 4000, 3], 6, 2, F16, True, 2500, True),
    "prefix_full": ([40, 1, 0, 99], [40, 17, 3, 0], 2, 2, F16, False, 63, False),
    "prefix_one_sequence": ([3], [30], 8, 1, BF16, True, 2000, False),
    "prefix_more_queries_than_keys": ([200, 4], [20, 1], 2, 1, BF16, True, 70, False),
}


@pytest.mark.parametrize("name", CASES)
def test_matches_the_oracle(name):
    nq, nk, H, Hk, dtype, causal, prefix, cache = CASES[name]
    b = Batch(nq, nk, H, Hk, dtype, causal, prefix, cache, seed=len(name))
    got = b.run()
    b.check(got)
    # a bound on the queries that is unknown or too low changes the tiles only
    for max_q in (0, 1):
        b.check(b.run(b.plan(max_q=max_q)))
    assert b.plan().flags() == 0


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_peaked_scores(dtype):
    b = Batch([90, 1, 1], [90, 400, 3000], 4, 2, dtype, scale=20.0)
    b.check(b.run())


def test_scale_argument_and_strided_views():
    g = torch.Generator().manual_seed(5)
    H, Hk = 6, 2
    b = Batch([100, 30], [100, 30], H, Hk, BF16)
    fused = torch.randn(130, H + 2 * Hk, 128, generator=g).to(BF16).cuda()
    b.q, b.k, b.v = fused[:, :H], fused[:, H:H + Hk], fused[:, H + Hk:]
    out = torch.empty(H, 130, 128, dtype=BF16, device="cuda").transpose(0, 1)
    got = b.run(out=out, sm_scale=0.2)
    assert got[0] is out
    b.check(got, sm=0.2)
    c = Batch([100, 30], [100, 30], H, Hk, BF16)
    c.q, c.k, c.v = (x.contiguous() for x in (b.q, b.k, b.v))
    same = c.run(sm_scale=0.2)
    assert torch.equal(same[0], out) and torch.equal(same[1], got[1])


@pytest.mark.parametrize("nq,nk,prefix", [([130, 1, 40], [130, 3000, 40], 0), ([1] * 9, [70] * 9, 300), ([150, 3], [150, 3], 100)])
def test_results_in_the_place_of_the_queries(nq, nk, prefix):
    b = Batch(nq, nk, 4, 2, BF16, prefix=prefix)
    want = b.run()
    got = b.run(out=b.q)
    assert got[0] is b.q and torch.equal(b.q, want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("heads_first", [False, True])
def test_results_beside_the_inputs_in_one_buffer(heads_first):
    b = Batch([100, 30], [100, 30], 4, 2, BF16)
    want = b.run()
    buf = torch.empty((12, 130, 128) if heads_first else (130, 12, 128), dtype=BF16, device="cuda")
    rows = buf.transpose(0, 1) if heads_first else buf
    q, k, out, v = rows.split((4, 2, 4, 2), 1)
    for to, x in ((q, b.q), (k, b.k), (v, b.v)):
        to.copy_(x)
    b.q, b.k, b.v = q, k, v
    got = b.run(out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_prefix_with_strides_of_its_own():
    b = Batch([1] * 5 + [90], [3, 70, 1, 9, 64, 90], 4, 2, F16, prefix=200)
    want = b.run()
    both = torch.stack((b.pk, b.pv), 1)            # [200, 2, Hk, 128]
    b.pk, b.pv = both[:, 0], both[:, 1]
    got = b.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rows_of_no_sequence_stay():
    b = Batch([3, 70, 1], [9, 70, 500], 4, 2, BF16)
    rows = b.qo[-1]
    q = torch.cat((b.q[:6], b.q, b.q[:11]))
    plan = ops.plan_packed_attn(ints(o + 6 for o in b.qo), ints(b.ko), rows + 17, b.k.shape[0], 4, 2, max_q=70)
    out = torch.full_like(q, 7.0)
    ops.packed_attn_fwd(q, b.k, b.v, plan, out=out)
    want = b.run()[0]
    assert torch.equal(out[6:6 + rows], want) and (out[:6] == 7).all() and (out[6 + rows:] == 7).all()
    # with a prefix whose pass runs over the rows of all sequences
    b = Batch([1] * 6, [2, 3, 4, 5, 6, 7], 4, 2, BF16, prefix=100)
    want = b.run()[0]
    q = torch.full((20, 4, 128), float("nan"), dtype=BF16, device="cuda")
    q[9:15] = b.q
    plan = ops.plan_packed_attn(ints(o + 9 for o in b.qo), ints(b.ko), 20, b.k.shape[0], 4, 2, prefix=100, max_q=1)
    out = torch.full_like(q, 7.0)
    ops.packed_attn_fwd(q, b.k, b.v, plan, out=out, prefix_k=b.pk, prefix_v=b.pv)
    assert (out[:9] == 7).all() and (out[15:] == 7).all()
    assert float((out[9:15].float() - want.float()).abs().max()) < 0.02


def test_shared_and_unordered_key_ranges():
    """Two sequences over the same cached keys, a third over a range behind and before theirs."""
    b = Batch([1, 4, 40], [300, 300, 64], 4, 2, F16, cache=False)
    k, v = b.k[:400], b.v[:400]
    plan = ops.plan_packed_attn(ints(b.qo), ints([100, 100, 7]), 45, 400, 4, 2, k_lens=ints([300, 300, 64]))
    got = ops.packed_attn_fwd(b.q, k, v, plan, return_lse=True)
    O, lse = orc.attention(*(x.float().cpu().numpy() for x in (b.q, k, v)), b.qo, [100, 100, 7], SM, True, [300, 300, 64])
    assert np.abs(got[0].float().cpu().numpy() - O).max() < 4e-3 and np.abs(got[1].cpu().numpy() - lse).max() < 1e-4
    assert plan.flags() == 0


@pytest.mark.parametrize("nq,nk,prefix", [([128, 40], [128, 40], 0), ([1, 1], [70, 5], 0), ([50, 9], [80, 9], 100),
                                          ([40, 9], [200, 9], 0), ([10, 70], [10, 70], 40)])   # the last two: waves without rows
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_keys_and_values_that_a_row_does_not_see_may_hold_anything(nq, nk, prefix, what, dtype):
    b = Batch(nq, nk, 2, 1, dtype, prefix=prefix)
    clean, W = b.run(), b.oracle(absolute=True)[0]
    b.k[b.ko[1] - 1, :, 3] = what      # the last key of sequence 0: seen by its last query alone
    b.v[b.ko[1] - 1, :, 17] = what
    got = b.run()
    last = b.qo[1] - 1
    rows = [r for r in range(b.qo[-1]) if r != last]
    near(got, clean, W, rows)


@pytest.mark.parametrize("nq,nk,H,Hk,prefix", [([2], [2], 128, 1, 0), ([3, 1], [70, 5], 256, 2, 0), ([3], [3], 200, 1, 0),
                                               ([2, 2, 2], [9, 66, 2], 128, 1, 100), ([5], [66], 129, 1, 0)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_unseen_keys_may_hold_anything_where_a_token_fills_a_tile(nq, nk, H, Hk, prefix, what):
    """With 128 query heads per key head or more, the rows of a tile may all belong to one token and see the same keys,
    while its last block holds keys of later tokens."""
    b = Batch(nq, nk, H, Hk, BF16, prefix=prefix)
    clean, W = b.run(), b.oracle(absolute=True)[0]
    b.k[b.ko[1] - 1, :, 3] = what      # the last key of sequence 0: seen by its last query alone
    b.v[b.ko[1] - 1, :, 17] = what
    got = b.run()
    near(got, clean, W, [r for r in range(b.qo[-1]) if r != b.qo[1] - 1])


@pytest.mark.parametrize("nq,nk", [([100], [100]), ([40, 9], [200, 9]), ([300, 1], [300, 700])])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_row_is_the_same_whatever_others_see(nq, nk, dtype):
    """The last token of sequence 0, its query, key and value (all finite): no bit of another row changes."""
    b = Batch(nq, nk, 4, 2, dtype)
    clean = b.run()
    last = b.qo[1] - 1
    b.q[last], b.k[b.ko[1] - 1], b.v[b.ko[1] - 1] = 3.0, 3.0, 50.0
    got = b.run()
    rows = [r for r in range(b.qo[-1]) if r != last]
    assert torch.equal(got[0][rows], clean[0][rows]) and torch.equal(got[1][:, rows], clean[1][:, rows])
    assert (got[0][last] == 50).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("prefix", [0, 1000])
def test_a_row_is_the_same_whatever_other_requests_and_heads_ask(prefix, dtype):
    b = Batch([1] * 40, list(range(180, 220)), 8, 2, dtype, prefix=prefix)
    clean = b.run()
    b.q[3, 1] = 8 * (b.pk[900, 0] if prefix else b.k[b.ko[4] - 1, 0])   # one head of one request, along one late key
    got = b.run()
    same = torch.ones(40, 8, dtype=torch.bool, device="cuda")
    same[3, 1] = False
    assert torch.equal(got[0][same], clean[0][same]) and torch.equal(got[1].t()[same], clean[1].t()[same])
    assert not torch.equal(got[0][3, 1], clean[0][3, 1])


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype):
    b = Batch([100], [100], 2, 1, dtype)
    clean, W = b.run(), b.oracle(absolute=True)[0]
    for row, d, what in ((70, 5, float("inf")), (40, 90, float("-inf")), (96, 33, float("nan"))):
        b.v[row, 0, d] = what
    got = b.run()
    out = got[0]
    assert torch.isposinf(out[70:, :, 5]).all() and torch.isneginf(out[40:, :, 90]).all() and torch.isnan(out[96:, :, 33]).all()
    out[70:, :, 5], out[40:, :, 90], out[96:, :, 33] = clean[0][70:, :, 5], clean[0][40:, :, 90], clean[0][96:, :, 33]
    near(got, clean, W, list(range(100)))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_infinite_values_at_the_end_of_a_partial_block(dtype):
    """Seen by every row: infinite in every row, and not NaN from the rows of the tile behind them."""
    b = Batch([40, 9, 1], [70, 3, 500], 2, 1, dtype, causal=False, prefix=33)
    b.v[69, 0, 5], b.v[72, 0, 90], b.pv[32, 0, 7] = float("inf"), float("-inf"), float("inf")
    out = b.run()[0]
    assert torch.isposinf(out[:40, :, 5]).all() and torch.isneginf(out[40:49, :, 90]).all() and torch.isposinf(out[:, :, 7]).all()
    out[:40, :, 5], out[40:49, :, 90], out[:, :, 7] = 0, 0, 0
    assert torch.isfinite(out).all()


def test_logits_of_minus_infinity():
    """Keys whose logit is -inf carry no weight, also where a whole block or a row has nothing else."""
    b = Batch([1, 1, 2], [200, 64, 70], 2, 1, BF16)
    b.q.abs_()
    b.k[:130, :, 0] = float("-inf")           # sequence 0: two whole blocks and two keys
    b.k[200:264, :, 0] = float("-inf")        # sequence 1: every key
    got = b.run()
    b.check(got)
    assert torch.isneginf(got[1][:, 1]).all() and not got[0][1].any()


def test_a_row_that_holds_nan_stays_alone():
    b = Batch([40, 3], [40, 100], 2, 2, F16)
    clean, W = b.run(), b.oracle(absolute=True)[0]
    b.q[7, 1] = float("nan")
    got = b.run()
    assert torch.isnan(got[0][7, 1]).all()
    got[0][7, 1], got[1][1, 7] = clean[0][7, 1], clean[1][1, 7]
    near(got, clean, W, list(range(43)))


def test_offsets_and_lengths_out_of_range_are_clamped_and_flagged():
    b = Batch([5, 5, 5], [20, 20, 20], 2, 1, BF16)
    plan = ops.plan_packed_attn(ints([0, 9, 5, 900]), ints([0, 20, 40, 60]), 15, 60, 2, 1)
    assert plan.flags() == 1
    ops.packed_attn_fwd(b.q, b.k, b.v, plan)
    plan = ops.plan_packed_attn(ints(b.qo), ints([-8, 20, 1 << 30, 0]), 15, 60, 2, 1, k_lens=ints([70, -3, 20]))
    assert plan.flags() == 2
    out = ops.packed_attn_fwd(b.q, b.k, b.v, plan)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and not out[5:].any()


def test_a_plan_for_another_shape_writes_nothing():
    b = Batch([5, 5], [20, 20], 2, 1, BF16)
    plan = b.plan()
    other = ops.PackedPlan(plan.data, ops.PackedShape.from_buffer_copy(bytes(plan.shape)))
    other.shape.causal = 0
    out = torch.full_like(b.q, 3.0)
    ops.packed_attn_fwd(b.q, b.k, b.v, other, out=out)
    assert (out == 3).all()


def test_a_plan_for_another_shape_writes_nothing_whichever_field_differs():
    """A larger plan run as a smaller one would address rows that the tensors do not have.  The first pair of shapes has
    the same 32-bit hash under a common way of mixing the fields."""
    shapes = [(41, 3876, 171939, 0, 32, 8, 1, 280), (34, 277, 189076, 0, 32, 8, 1, 69)]
    base = (7, 300, 900, 64, 8, 4, 1, 50)
    pairs = [shapes] + [[base, base[:i] + (n,) + base[i + 1:]] for i, n in
                        enumerate((6, 299, 899, 63, 4, 2, 0, 49))]
    for made, run in pairs:
        n, tq, tk, prefix, H, Hk, causal, max_q = made
        qo = ints(np.linspace(0, tq, n + 1).astype(int))
        plan = ops.plan_packed_attn(qo, ints(np.linspace(0, tk, n + 1).astype(int)), tq, tk, H, Hk, causal=causal, prefix=prefix,
                                    max_q=max_q)
        shape = ops.PackedShape(*run[:6], 128, *run[6:])
        other = ops.PackedPlan(torch.zeros(plan.data.numel() + (1 << 20), dtype=torch.uint8, device="cuda"), shape)
        at = [ops._aligned(p.data) - p.data.data_ptr() for p in (plan, other)]
        other.data[at[1]:at[1] + plan.plan_bytes] = plan.data[at[0]:at[0] + plan.plan_bytes]
        assert other.plan_bytes <= other.data.numel() - 256
        q, k = (torch.zeros(dims, dtype=BF16, device="cuda") for dims in (other.q_dims, other.k_dims))
        pk = torch.zeros(other.prefix_dims, dtype=BF16, device="cuda") if run[3] else None
        out = torch.full_like(q, 3.0)
        ops.packed_attn_fwd(q, k, k, other, prefix_k=pk, prefix_v=pk, out=out)
        assert (out == 3).all(), (made, run)


def test_deterministic_and_the_plan_can_be_written_again():
    b = Batch([1] * 30 + [300], [int(x) for x in np.linspace(1, 4000, 30)] + [300], 8, 2, BF16, cache=True)
    plan = b.plan()
    a = b.run(plan)
    for _ in range(3):
        again = b.run(b.plan(out=plan))
        assert torch.equal(a[0], again[0]) and torch.equal(a[1], again[1])


def test_captured_with_lengths_that_change():
    """Plan and attention in one graph; the lengths on the device change between replays."""
    b = Batch([1] * 6, [900, 30, 64, 1, 500, 77], 8, 2, F16, prefix=300, cache=True)
    b.k.nan_to_num_(0.5)
    b.v.nan_to_num_(0.25)
    qo, ko, nk = ints(b.qo), ints(b.ko), ints(b.nk)
    plan = b.plan()
    out = torch.empty_like(b.q)

    def step():
        ops.plan_packed_attn(qo, ko, 6, b.k.shape[0], 8, 2, k_lens=nk, prefix=300, max_q=1, out=plan)
        return ops.packed_attn_fwd(b.q, b.k, b.v, plan, prefix_k=b.pk, prefix_v=b.pv, out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([900, 30, 64, 1, 500, 77], [1, 2, 3, 4, 5, 6], [0, 907, 0, 64, 65, 128], [900, 30, 64, 1, 500, 77]):
        nk.copy_(ints(lens))
        b.nk = lens
        want = b.run()[0].clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_streams_with_one_plan():
    b = Batch([1] * 5, [3000, 10, 700, 64, 1], 8, 2, BF16, cache=True)
    plan = b.plan()
    want = b.run(plan)[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(ops.packed_attn_fwd(b.q, b.k, b.v, plan))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes; the sequences stand at its ends."""
    Hk, rows = 8, 2_300_000                       # 4.7 GB for each of K and V
    k = torch.zeros(rows, Hk, 128, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    b = Batch([1, 70], [300, 200], 16, Hk, BF16, cache=True)
    at = [0, rows - 200]
    for i in range(2):
        k[at[i]:at[i] + b.nk[i]] = b.k[b.ko[i]:b.ko[i] + b.nk[i]]
        v[at[i]:at[i] + b.nk[i]] = b.v[b.ko[i]:b.ko[i] + b.nk[i]]
    plan = ops.plan_packed_attn(ints(b.qo), ints(at), 71, rows, 16, Hk, k_lens=ints(b.nk), max_q=70)
    got = ops.packed_attn_fwd(b.q, k, v, plan, return_lse=True)
    torch.cuda.synchronize()
    b.check(got)


def test_no_queries_and_no_keys():
    q = torch.empty(0, 4, 128, dtype=F16, device="cuda")
    k = torch.empty(5, 2, 128, dtype=F16, device="cuda")
    plan = ops.plan_packed_attn(ints([0, 0]), ints([0, 5]), 0, 5, 4, 2)
    assert ops.packed_attn_fwd(q, k, k, plan).shape == (0, 4, 128)
    q, k = torch.ones(3, 4, 128, dtype=F16, device="cuda"), k[:0]
    plan = ops.plan_packed_attn(ints([0, 3]), ints([0, 0]), 3, 0, 4, 2)
    out, lse = ops.packed_attn_fwd(q, k, k, plan, return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()


def test_many_sequences():
    n = 3000
    rng = np.random.default_rng(1)
    nq, nk = rng.integers(0, 3, n), rng.integers(0, 40, n)
    b = Batch(nq, nk, 2, 1, F16)
    b.check(b.run())


def test_norm_rotation_and_attention_of_a_layer():
    """Two requests of different grids: fused projection -> norm and rotation in place -> packed attention, and the
    next token of each against the caches; every step against the float64 oracles run on the step's own inputs."""
    from oracle import rotary as orot
    H, Hk, n = 4, 2, [150, 77]
    g = torch.Generator().manual_seed(4)
    fused = torch.randn(sum(n), H + 2 * Hk, 128, generator=g).to(BF16).cuda()
    raw = fused.clone()
    q, k, v = fused[:, :H], fused[:, H:H + Hk], fused[:, H + Hk:]
    pos = torch.cat([torch.stack([torch.arange(m) // 50, torch.arange(m) // 10 % 5, torch.arange(m) % 10]) for m in n], 1)
    rot = ops.RotaryAxes((22, 21, 21))
    w = (1 + 0.1 * torch.randn(128, generator=g)).cuda()
    ops.qk_norm_rope(q[None], k[None], rotary=rot, positions=pos.to(torch.int32).cuda(), norm="head", q_weight=w, k_weight=w,
                     q_out=q[None], k_out=k[None])
    for x, r in ((q, raw[:, :H]), (k, raw[:, H:H + Hk])):
        want = orot.norm_rotate(r.float().cpu().numpy()[None], "head", w.cpu().numpy(), 1e-6, pos.numpy(), rot.pairs, rot.freqs)[0]
        assert (np.abs(x.float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16).all()
    b = Batch(n, n, H, Hk, BF16)
    b.q, b.k, b.v = q, k, v
    b.check(b.run())


def test_refusals_of_the_binding():
    b = Batch([5, 3], [9, 3], 4, 2, F16)
    plan = b.plan()

    def no(match, **kw):
        a = dict(q=b.q, k=b.k, v=b.v, plan=plan) | kw
        with pytest.raises(ValueError, match=match):
            ops.packed_attn_fwd(**a)

    no("q must be", q=b.q[:7])
    no("k must be", k=b.k.to(BF16))
    no("v must be", v=b.v[:, :1])
    no("prefix has 0 rows", prefix_k=b.k, prefix_v=b.v)
    no("out must be", out=b.q[:, :2])
    no("share memory", out=b.q[:1].expand(8, 4, 128))
    no("contiguous", q=torch.empty(8, 4, 256, dtype=F16, device="cuda")[:, :, ::2])
    with pytest.raises(TypeError):
        ops.packed_attn_fwd(b.q.float(), b.k.float(), b.v.float(), plan)
    with pytest.raises(RuntimeError, match="out overlaps k"):
        full = Batch([9], [9], 2, 2, F16)
        ops.packed_attn_fwd(full.q, full.k, full.v, full.plan(), out=full.k)
    with pytest.raises(ValueError, match="another shape"):
        ops.plan_packed_attn(ints(b.qo), ints(b.ko), 8, 12, 4, 2, causal=False, out=plan)
    with pytest.raises(ValueError, match="int32 vector"):
        ops.plan_packed_attn(ints(b.qo).long(), ints(b.ko), 8, 12, 4, 2)
    with pytest.raises(ValueError, match="entries"):
        ops.plan_packed_attn(ints(b.qo), ints(b.ko[:2]), 8, 12, 4, 2)
    with pytest.raises(RuntimeError, match="multiple"):
        ops.plan_packed_attn(ints(b.qo), ints(b.ko), 8, 12, 4, 3)
