"""Packed prompts where numbers run out: scores that are not finite, values near the end of their range, scores that the tensor
cores add up exactly, and calls at the edge of what the header allows."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2412_20105_b200 import binding as B
from paper_2412_20105_b200.build import build
from test_gpu_packed import INVALID, _attend, _check_attend, _desc, _f64, _i32, _inputs, _starts

gpu = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- scores that are not finite
@gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", ["nan key", "inf score"])
def test_one_bad_key_reaches_every_later_row_wherever_it_stands(dim, bad):
    """A NaN score, or one of +Inf, makes its row NaN; rows ahead of the key keep their bits."""
    lens = [420]
    q, k, v = _inputs(lens, 2, 1, dim, layout="dense", seed=dim)
    q[..., 1] = q[..., 1].abs() + 1
    clean, lse = _attend(q, k, v, lens)
    for at in list(range(34)) + [63, 64, 100, 127, 128, 133, 255, 300]:
        k2 = k.clone()
        if bad == "nan key":
            k2[at] = float("nan")
        else:
            k2[at, 0, 1] = float("inf")
        out, sums = _attend(q, k2, v, lens)
        assert torch.equal(out[:at], clean[:at]) and torch.equal(sums[:, :at], lse[:, :at]), at
        assert torch.isnan(out[at:]).all() and torch.isnan(sums[:, at:]).all(), at


@gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("first,last", [(0, 1), (3, 6), (36, 46), (100, 101), (0, 64), (0, 200)])
def test_scores_of_minus_infinity_have_no_weight(dim, first, last):
    """Keys first .. last - 1 score -Inf.  A row that sees no others has no softmax; the rest come out as without them."""
    n = 420
    q, k, v = _inputs([n], 2, 1, dim, layout="dense", seed=dim + first)
    q[..., 1] = q[..., 1].abs() + 1
    k[first:last, 0, 1] = float("-inf")
    out, sums = _attend(q, k, v, [n])
    none = last if first == 0 else 0
    assert torch.isnan(out[:none]).all() and bool((sums[:, :none] == -math.inf).all())
    kn, vn, qn = _f64(k[:, 0]), _f64(v[:, 0]), _f64(q)
    kn[first:last] = 0.0
    for i in list(range(none, n, 17)) + [n - 1]:
        stay = [j for j in range(i + 1) if not first <= j < last]
        for h in range(2):
            x = kn[stay] @ qn[i, h] / math.sqrt(dim)
            p = np.exp(x - x.max())
            ref, spread = p @ vn[stay] / p.sum(), p @ np.abs(vn[stay]) / p.sum()
            # as in _check_attend
            logit = 2.0 ** -20 * (1 + float((np.abs(kn[stay]) @ np.abs(qn[i, h])).max()) / math.sqrt(dim))
            assert np.all(np.abs(_f64(out[i, h]) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * logit) * spread + 1e-30), (i, h)
            total = math.log(p.sum()) + x.max()
            assert abs(float(sums[h, i]) - total) <= 2 * logit + 2.0 ** -23 * abs(total), (i, h)


@gpu
@pytest.mark.parametrize("copies", [1, 40])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_bad_query_reaches_every_key_it_sees(copies, dim):
    """A NaN query has a NaN lse: every key up to it has received NaN, whatever column the query stands in.  One prompt (items
    shared by blocks) and many (whole items)."""
    n = 300
    lens = [n] * copies
    q, k, v = _inputs(lens, 2, 1, dim, layout="dense", seed=dim)
    _, lse = _attend(q, k, v, lens)
    clean = torch.full((copies, 1, 320), -1.0, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), clean)
    for at in list(range(128, 162)) + [0, 22, 127, 255, 256, 282, n - 1]:
        for kind in ("both", "lse", "query"):
            q2, lse2, w = q.clone(), lse.clone(), torch.full_like(clean, -1.0)
            if kind != "lse":
                q2[at] = float("nan")
            if kind != "query":
                lse2[:, at] = float("nan")
            B.packed_weights(q2, k, lse2, _starts(lens), w)
            assert torch.isnan(w[0, 0, :at + 1]).all(), (at, kind)
            assert torch.equal(w[0, 0, at + 1:], clean[0, 0, at + 1:]) and torch.equal(w[1:], clean[1:]), (at, kind)


@gpu
@pytest.mark.parametrize("window", list(range(1, 33)) + [64, 80])
def test_one_bad_key_has_received_nan(window):
    """The last key is seen by the last query only, which stands in column window - 1 of its tile."""
    n = 200
    q, k, v = _inputs([n], 2, 1, 64, layout="dense", seed=window)
    _, lse = _attend(q, k, v, [n])
    k[n - 1] = float("nan")
    w = torch.full((1, 1, 256), -1.0, device="cuda")
    B.packed_weights(q, k, lse, _starts([n]), w, window)
    assert torch.isnan(w[0, 0, n - 1]) and torch.isfinite(w[0, 0, :n - 1]).all() and bool((w[0, 0, n:] == -1).all())


# ------------------------------------------------------------------------------------------------ the ends of the range
@gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_large_values_behind_scores_that_grow(dim):
    """Scores rise by 40 (2^57.7 in weight) behind the first keys, and the values that they meet are near 10^20."""
    n = 400
    q, k, v = _inputs([n], 2, 1, dim, layout="dense", seed=dim)
    k *= 0.01
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[96:, 0, 0] = 5 * math.sqrt(dim)
    v *= 1e20
    out, lse = _attend(q, k, v, [n])
    _check_attend(q, k, v, [n], out, lse)


# --------------------------------------------------------------------------------------------------- sums that are exact
@gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_weights_of_scores_that_the_tensor_core_adds_up_exactly(dim):
    """All of a score lies in one dim, so its sum is exact, and lse is 0.  Scores near -50 show what multiplies them."""
    n = 512
    q, k = (torch.zeros(n, 1, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    build()
    g = torch.Generator().manual_seed(dim)
    q[:, 0, 5] = 64.0
    k[:, 0, 5] = ((torch.rand(n, generator=g) * 0.2 - 1) * (50.0 * math.sqrt(dim) / 64)).bfloat16().cuda()
    w = torch.zeros(1, 1, n, device="cuda")
    B.packed_weights(q, k, torch.zeros(1, n, device="cuda"), _i32([0, n]), w, 1)
    want = np.exp(_f64(k[:, 0, 5]) * 64.0 / math.sqrt(dim))
    # the exponent of 2 is at most 72.2: log2(e) / sqrt(D) rounded to 32 bits (half a step, 2^-24 of it), one fma (half a step at
    # 64 .. 128, 2^-18), both times ln 2; exp2 and its sum with zeros 2^-21
    bound = math.log(2) * (72.2 * 2.0 ** -24 + 2.0 ** -18) + 2.0 ** -21
    err = _f64(w[0, 0]) / want - 1
    assert np.abs(err).max() <= bound, (float(np.abs(err).max()), bound)


# --------------------------------------------------------------------------------------------------- calls at the edge
def test_nothing_to_do_needs_no_pointers():
    """Empty tensors have the address 0."""
    build()
    lib = B.load()
    for kw in (dict(total=0), dict(num_seqs=0), dict(total=0, num_seqs=0)):
        d = _desc(**kw)
        assert lib.st3_packed_weights(C.byref(d), None, None, None, 4096, None, 128, 0, None, None) == 0
        assert lib.st3_packed_attend(C.byref(d), None, None, None, 4096, None, None, None, None) == 0
    d = _desc()
    assert lib.st3_packed_weights(C.byref(d), 4096, 4096, None, 4096, 4096, 128, 0, None, None) == INVALID
    assert lib.st3_packed_weights(C.byref(d), 4096, 4096, 4096, 4096, None, 128, 0, None, None) == INVALID


@gpu
@pytest.mark.parametrize("total,seqs", [(0, 3), (20, 0), (0, 0)])
def test_batches_of_no_tokens_or_no_sequences(total, seqs):
    q, k, v = _inputs([total], 4, 2, 64, layout="dense")
    cu = _i32([0] * (seqs + 1))
    out, lse = torch.full_like(q, 3.0), torch.full((4, total), 3.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.packed_attend(q, k, v, cu, out, lse, status)
    w = torch.full((seqs, 2, 64), 3.0, device="cuda")
    B.packed_weights(q, k, lse, cu, w, 0, status)
    assert int(status) == 0 and bool((out == 3).all()) and bool((lse == 3).all()) and bool((w == 3).all())


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses stand in for tensors")
@pytest.mark.parametrize("kw", [dict(num_kv_heads=1, k_head_stride=0, v_head_stride=4), dict(total=1, q_token_stride=0, out_token_stride=3),
                                dict(total=1, k_token_stride=-1, v_token_stride=1),
                                dict(num_heads=1, num_kv_heads=1, q_head_stride=0, k_head_stride=-5, v_head_stride=1, out_head_stride=2)])
def test_a_stride_that_is_never_used_may_be_anything(kw):
    """One head, or one token: what torch calls its stride says nothing.  Without a GPU the call gets as far as the driver."""
    build()
    lib, d = B.load(), _desc(**kw)
    assert lib.st3_packed_attend(C.byref(d), 4096, 4096, 4096, 4096, 4096, None, None, None) != INVALID
    assert lib.st3_packed_weights(C.byref(d), 4096, 4096, 4096, 4096, 4096, 128, 0, None, None) != INVALID


@gpu
def test_one_head_or_one_token_with_strides_of_any_kind():
    lens = [70, 30]
    q, k, v = _inputs(lens, 3, 1, 64, layout="dense")
    want, lse = _attend(q, k, v, lens)
    odd = lambda x, token, head: x.as_strided(x.shape, (x.stride(0) if token is None else token, x.stride(1) if head is None else head, 1))
    out = torch.zeros_like(q)
    got, sums = _attend(q, odd(k, None, 0), odd(v, None, 5), lens, out=out)
    assert torch.equal(got, want) and torch.equal(sums, lse)
    w, w2 = torch.zeros(2, 1, 128, device="cuda"), torch.zeros(2, 1, 128, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), w)
    B.packed_weights(q, odd(k, None, 1), lse, _starts(lens), w2)
    assert torch.equal(w, w2)
    one = [x[:1].contiguous() for x in (q, k, v)]
    got, sums = _attend(odd(one[0], 0, None), odd(one[1], 3, None), odd(one[2], 1, None), [1], out=odd(torch.zeros_like(one[0]), 7, None))
    assert torch.equal(got, v[:1].expand(1, 3, 64)) and torch.isfinite(sums).all()


@gpu
@pytest.mark.parametrize("cu", [[0, 128, 127, 256], [0, 256, 255, 256], [0, 200, 100, 256], [0, 256, 0, 256], [300, 300, 300, 300],
                                [256, 0, 0, 256], [0, 100, 256, 257], [2 ** 31 - 1, 0, 128, 256]])
def test_every_kind_of_wrong_offsets_is_reported(cu):
    """Also where no item falls to the sequence that is wrong."""
    for heads, kv in ((2, 1), (1, 1)):
        q, k, v = _inputs([256], heads, kv, 64, layout="dense")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.packed_attend(q, k, v, _i32(cu), torch.zeros_like(q), None, status)
        assert int(status) == B.DEV_RANGE, heads
        status.zero_()
        B.packed_weights(q, k, torch.zeros(heads, 256, device="cuda"), _i32(cu), torch.zeros(3, kv, 256, device="cuda"), 0, status)
        assert int(status) == B.DEV_RANGE, heads


@gpu
def test_one_wrong_sequence_among_thousands_is_reported():
    q, k, v = _inputs([4000], 2, 1, 64, layout="dense")
    for b in (0, 31, 32, 1999, 3998):
        cu = torch.arange(4001, dtype=torch.int32)
        cu[b + 1] -= 2                             # that sequence has -1 tokens, the next one three
        if b == 3998:
            cu[4000] = 4001
        for weights in (False, True):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            if weights:
                B.packed_weights(q, k, torch.zeros(2, 4000, device="cuda"), cu.cuda(), torch.zeros(4000, 1, 64, device="cuda"), 0, status)
            else:
                B.packed_attend(q, k, v, cu.cuda(), torch.zeros_like(q), None, status)
            assert int(status) == B.DEV_RANGE, (b, weights)


@gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("score", [-200.0, float("-inf")])
def test_a_score_far_below_leaves_nothing_of_a_large_value(dim, score):
    """e^-200 times 10^30 is nothing beside values of 10^-10, wherever the key stands."""
    n = 420
    q, k, v = _inputs([n], 2, 1, dim, layout="dense", seed=dim)
    k *= 0.01
    q[..., 0], k[..., 0] = 8.0, 0.0
    v *= 1e-10
    for at in list(range(8)) + [68, 69, 101]:
        k2, v2 = k.clone(), v.clone()
        k2[at, 0, 0] = score * math.sqrt(dim) / 8
        v2[at] = 1e30
        out, _ = _attend(q, k2, v2, [n])
        rows = list(range(at + 1, n, 37))
        qn, kn, vn = _f64(q), _f64(k2[:, 0]), _f64(v2[:, 0])
        for i in rows:
            stay = [j for j in range(i + 1) if j != at]
            for h in range(2):
                x = kn[stay] @ qn[i, h] / math.sqrt(dim)
                p = np.exp(x - x.max())
                want, spread = p @ vn[stay] / p.sum(), p @ np.abs(vn[stay]) / p.sum()
                logit = 2.0 ** -20 * (1 + float((np.abs(kn[stay]) @ np.abs(qn[i, h])).max()) / math.sqrt(dim))
                bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * logit) * spread + 1e-30
                assert np.all(np.abs(_f64(out[i, h]) - want) <= bound), (at, i, h)
