"""Packed prompts with grouped heads (causal attention, weights received) through the C ABI against the fp64 oracle, and the
way of a batch through prompt, cache, decode steps and evictions."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2412_20105_b200 import binding as B
from paper_2412_20105_b200.build import build

gpu = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(lens):
    return _i32([0] + list(np.cumsum(lens)))


def _inputs(lens, heads, kv, dim, seed=0, layout="fused"):
    build()
    g = torch.Generator().manual_seed(seed)
    total = sum(lens)
    qkv = [torch.randn(total, n, dim, generator=g).bfloat16().cuda() for n in (heads, kv, kv)]
    if layout == "fused":
        qkv = list(torch.cat(qkv, 1).split([heads, kv, kv], 1))
    elif layout == "head first":
        qkv = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in qkv]
    return qkv


def _f64(x):
    return x.double().cpu().numpy()


def _attend(q, k, v, lens, lse=True, out=None):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    sums = torch.full((q.shape[1], q.shape[0]), float("nan"), device="cuda") if lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.packed_attend(q, k, v, _starts(lens), out, sums, status)
    assert int(status) == 0
    return out, sums


def _check_attend(q, k, v, lens, out, lse):
    ref, sums, spread, reach = O.packed_attend(_f64(q), _f64(k), _f64(v), lens)
    # P enters the second product as bf16 (half a step, 2^-8 of a term at most), the output is rounded to bf16 as well; logits
    # are exact products summed in fp32 (2^-20 of the largest sum of magnitudes), exp2 and sums are good to 2^-20
    logit = 2.0 ** -20 * (reach + 1)
    bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * logit.T[:, :, None]) * spread + 1e-30
    err = np.abs(_f64(out) - ref)
    assert np.all(err <= bound), float((err - bound).max())
    if lse is not None:
        assert np.all(np.abs(_f64(lse) - sums) <= 2 * logit + 2.0 ** -23 * np.abs(sums))
    return ref, sums, reach


SHAPES = [([1], 2, 1, 128), ([1, 37, 130], 8, 2, 64), ([128], 4, 4, 128), ([129, 127, 128], 4, 2, 128), ([0, 5, 0, 0, 64, 0], 6, 1, 64),
          ([257, 256, 255], 3, 1, 128), ([300, 1, 511, 513], 5, 5, 64), ([675, 640], 8, 2, 128), ([1100], 14, 2, 128),
          ([3] * 90 + [200], 4, 1, 64), ([200, 65], 1, 1, 64), ([130], 16, 1, 128)]


@gpu
@pytest.mark.parametrize("lens,heads,kv,dim", SHAPES)
@pytest.mark.parametrize("layout", ["fused", "dense", "head first"])
def test_attention_of_packed_prompts(lens, heads, kv, dim, layout):
    q, k, v = _inputs(lens, heads, kv, dim, seed=sum(lens), layout=layout)
    out, lse = _attend(q, k, v, lens)
    _check_attend(q, k, v, lens, out, lse)


@gpu
@pytest.mark.parametrize("lens,heads,kv,dim", SHAPES)
@pytest.mark.parametrize("window", [0, 1, 32, 200])
def test_weights_received(lens, heads, kv, dim, window):
    q, k, _ = _inputs(lens, heads, kv, dim, seed=sum(lens) + 1)
    _, sums, _, reach = O.packed_attend(_f64(q), _f64(k), np.zeros((sum(lens), kv, dim)), lens)
    lse = torch.tensor(sums, dtype=torch.float32, device="cuda")
    cap = -(-max(lens) // 64) * 64
    w = torch.full((len(lens), kv, cap), -3.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), w, window, status)
    assert int(status) == 0
    want = O.packed_weights(_f64(q), _f64(k), _f64(lse), lens, window)
    # logits and sums as above, lse's product with log2(e) in fp32, and a chain of additions of n * group positive terms
    rel = 2.0 ** -18 * (1 + float(reach.max()) + float(np.abs(sums).max()))
    for b, n in enumerate(lens):
        got = _f64(w[b])
        assert np.all(np.abs(got[:, :n] - want[b]) <= rel * want[b] + 1e-30)
        assert np.all(got[:, n:] == -3.0)


@gpu
def test_logits_far_apart_and_growing_along_the_row():
    """The running reference moves (later keys are larger by more than 2^32) and small terms vanish."""
    lens, dim = [700], 64
    q, k, v = _inputs(lens, 2, 1, dim, layout="dense")
    k *= torch.linspace(0, 40, 700, device="cuda")[:, None, None].bfloat16()
    q.abs_()
    k.abs_()
    k[300] = 0
    out, lse = _attend(q, k, v, lens)
    _check_attend(q, k, v, lens, out, lse)
    q.neg_()                                     # and falling
    out, lse = _attend(q, k, v, lens)
    _check_attend(q, k, v, lens, out, lse)


@gpu
def test_sequences_do_not_reach_into_each_other():
    """Every sequence but one is NaN and Inf: its rows come out as they do alone."""
    lens = [70, 200, 3, 131, 128]
    for heads, kv, dim in ((4, 2, 128), (3, 1, 64)):
        q, k, v = _inputs(lens, heads, kv, dim, layout="dense")
        clean, _ = _attend(q, k, v, lens)
        at = np.cumsum([0] + lens)
        for s in range(len(lens)):
            mine = torch.zeros(sum(lens), dtype=torch.bool, device="cuda")
            mine[at[s]:at[s + 1]] = True
            bad = [torch.where(mine[:, None, None], x, torch.full_like(x, y)) for x, y in ((q, float("nan")), (k, float("inf")), (v, float("nan")))]
            out, lse = _attend(*bad, lens)
            assert torch.equal(out[mine], clean[mine]), s
            w = torch.zeros(len(lens), kv, 256, device="cuda")
            B.packed_weights(bad[0], bad[1], lse, _starts(lens), w)
            assert torch.isfinite(w[s]).all()
            assert math.isclose(float(w[s, :, :lens[s]].sum()), heads * lens[s], rel_tol=1e-4)


@gpu
def test_keys_in_the_future_may_be_anything():
    lens = [260]
    q, k, v = _inputs(lens, 2, 2, 128, layout="dense")
    clean, lse = _attend(q, k, v, lens)
    k[200:] = float("nan")
    out, sums = _attend(q, k, v, lens)
    assert torch.equal(out[:200], clean[:200]) and torch.equal(sums[:, :200], lse[:, :200])
    assert torch.isnan(out[200:]).all() and torch.isnan(sums[:, 200:]).all()


@gpu
def test_outputs_with_strides_and_without_sums():
    lens = [100, 61]
    q, k, v = _inputs(lens, 4, 2, 64)
    want, _ = _attend(q, k, v, lens)
    for shape, view in (((161, 7, 64), lambda x: x[:, 2:6]), ((4, 170, 64), lambda x: x[:, 5:166].transpose(0, 1)),
                        ((161, 4, 72), lambda x: x[:, :, 8:])):
        room = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
        out = view(room)
        _attend(q, k, v, lens, lse=False, out=out)
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert bool((room == 7.0).all())         # nothing beside the view was written


@gpu
def test_rows_of_no_sequence_are_left_as_they_were():
    """A padded batch: tokens ahead of the first sequence and behind the last one, with anything in them."""
    lens, before, after = [100, 0, 61], 5, 200
    for heads, kv in ((4, 2), (3, 3)):
        q, k, v = _inputs(lens, heads, kv, 64, layout="dense")
        want, lse = _attend(q, k, v, lens)
        pad = lambda x: torch.cat([torch.full_like(x[:before], float("nan")), x, torch.full((after,) + x.shape[1:], float("inf"), dtype=x.dtype, device="cuda")])
        out = torch.full((before + 161 + after, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        sums = torch.full((heads, out.shape[0]), 7.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.packed_attend(pad(q), pad(k), pad(v), _starts(lens) + before, out, sums, status)
        assert int(status) == 0
        mine = slice(before, before + 161)
        assert torch.equal(out[mine], want) and torch.equal(sums[:, mine], lse)
        assert bool((out[:before] == 7).all()) and bool((out[before + 161:] == 7).all()) and bool((sums[:, before + 161:] == 7).all())
        w, w2 = torch.full((3, kv, 128), -1.0, device="cuda"), torch.full((3, kv, 128), -1.0, device="cuda")
        B.packed_weights(q, k, lse, _starts(lens), w)
        B.packed_weights(pad(q), pad(k), sums, _starts(lens) + before, w2, 0, status)
        assert torch.equal(w, w2) and int(status) == 0


@gpu
def test_thousands_of_sequences_most_of_them_empty():
    g = np.random.default_rng(5)
    lens = [int(x) for x in g.integers(0, 3, size=3001) * (g.random(3001) < 0.3)]
    q, k, v = _inputs(lens, 4, 2, 64, seed=8)
    out, lse = _attend(q, k, v, lens)
    _check_attend(q, k, v, lens, out, lse)
    w = torch.full((3001, 2, 64), -1.0, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), w)
    want = O.packed_weights(_f64(q), _f64(k), _f64(lse), lens)
    got = w.cpu().numpy()
    for s, n in enumerate(lens):   # logits and sums below 24 together: 2^-18 * (1 + 24) < 1e-4
        assert np.allclose(got[s, :, :n], want[s], rtol=1e-4) and np.all(got[s, :, n:] == -1)


@gpu
def test_offsets_that_are_not_ascending_are_reported():
    q, k, v = _inputs([64, 64, 64], 2, 1, 64, layout="dense")
    good, _ = _attend(q, k, v, [64, 64, 64])
    for cu in ([0, 64, 200, 192], [0, 64, 32, 192], [-5, 64, 128, 192], [0, 64, 128, 300]):
        out = torch.zeros_like(q)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.packed_attend(q, k, v, _i32(cu), out, None, status)
        assert int(status) == B.DEV_RANGE
    status.zero_()
    w = torch.zeros(3, 1, 32, device="cuda")
    B.packed_weights(q, k, torch.zeros(2, 192, device="cuda"), _i32([0, 64, 80, 192]), w, 0, status)    # longer than the capacity
    assert int(status) == B.DEV_RANGE and bool(w[1].any()) and not bool(w[0].any()) and not bool(w[2].any())


@gpu
def test_more_items_than_the_gpu_holds_and_a_long_sequence():
    """Sampled rows of a batch with one sequence of 5000 tokens, whose items last a hundred times the shortest ones'."""
    lens = [5000] + [int(x) for x in np.random.default_rng(0).integers(1, 300, size=40)]
    q, k, v = _inputs(lens, 8, 4, 128, seed=4)
    out, lse = _attend(q, k, v, lens)
    at = np.cumsum([0] + lens)
    qn, kn, vn = _f64(q), _f64(k), _f64(v)
    for s, i in [(0, 0), (0, 127), (0, 128), (0, 2559), (0, 4999), (7, 0), (40, lens[40] - 1), (20, lens[20] // 2)]:
        row = at[s] + i
        for h in (0, 3, 7):
            kk, vv = kn[at[s]:row + 1, h // 2], vn[at[s]:row + 1, h // 2]
            x = kk @ qn[row, h] / math.sqrt(128)
            p = np.exp(x - x.max())
            total = p.sum()
            ref, spread = p @ vv / total, p @ np.abs(vv) / total
            assert np.all(np.abs(_f64(out[row, h]) - ref) <= 2.0 ** -8 * (np.abs(ref) + spread * 1.01) + 1e-30), (s, i, h)
            assert abs(float(lse[h, row]) - (math.log(total) + x.max())) <= 1e-4
    w = torch.zeros(len(lens), 4, 5056, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), w)
    sums = w.sum(2).cpu().numpy()
    assert np.allclose(sums, np.array(lens)[:, None] * 2, rtol=1e-4)       # every row's probabilities add up to 1


@gpu
def test_same_bits_on_another_stream_and_in_a_graph():
    lens = [700, 33, 512, 129]
    q, k, v = _inputs(lens, 8, 2, 128)
    out, lse = _attend(q, k, v, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out2, lse2 = _attend(q, k, v, lens)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    cu, w = _starts(lens), torch.zeros(4, 2, 704, device="cuda")
    B.packed_weights(q, k, lse, cu, w)
    out3, lse3, w3 = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.packed_attend(q, k, v, cu, out3, lse3)
        B.packed_weights(q, k, lse3, cu, w3)
    graph.replay()
    assert torch.equal(out, out3) and torch.equal(w, w3)
    # other lengths of the same total, through the same graph
    other = [129, 512, 33, 700]
    cu.copy_(_starts(other))
    graph.replay()
    out4, lse4 = _attend(q, k, v, other)
    assert torch.equal(out3, out4) and torch.equal(lse3, lse4)


@gpu
def test_a_batch_from_prompt_to_decoding_with_evictions():
    """Prompts -> weights -> 8-bit cache -> cut to a budget -> decode steps that accumulate and evict, against the oracle."""
    lens, heads, kv, dim, keep, recent = [300, 97, 260], 8, 2, 128, 128, 16
    q, k, v = _inputs(lens, heads, kv, dim, seed=9)
    out, lse = _attend(q, k, v, lens)
    _check_attend(q, k, v, lens, out, lse)
    cache = B.Cache.empty(3, kv, dim, 320)
    cache.store(k, v, _starts(lens))
    B.packed_weights(q, k, lse, _starts(lens), cache.weights)
    oracle = [[O.Head(dim) for _ in range(kv)] for _ in lens]
    at = np.cumsum([0] + lens)
    held, seen = _i32(lens), _i32(lens)
    for b, row in enumerate(oracle):
        for h, o in enumerate(row):
            o.store(_f64(k[at[b]:at[b + 1], h]), _f64(v[at[b]:at[b + 1], h]))
    g = torch.Generator().manual_seed(5)
    for step in range(6):
        for b, row in enumerate(oracle):       # the oracle takes over the weights, so that both cut by the same ones
            for h, o in enumerate(row):
                o.weights = [float(x) for x in cache.weights[b, h, :len(o)]]
                o.evict(keep, recent, int(seen[b]))
        held = cache.evict(held, seen, keep, recent)
        assert held.tolist() == [len(r[0]) for r in oracle]
        kn, vn = (torch.randn(3, kv, dim, generator=g).bfloat16() for _ in range(2))
        qn = torch.randn(3, heads, dim, generator=g).bfloat16()
        cache.store(kn.cuda(), vn.cuda(), _starts([1, 1, 1]), start=held, pos=seen)
        for b, row in enumerate(oracle):
            for h, o in enumerate(row):
                o.store(_f64(kn[b:b + 1, h]), _f64(vn[b:b + 1, h]), int(seen[b]))
        held, seen = held + 1, seen + 1
        before = cache.weights.clone()
        got = torch.empty(3, heads, dim, dtype=torch.bfloat16, device="cuda")
        cache.attend(qn.cuda(), held, got, weights_out=cache.weights)
        ks, vs, ids, _ = (x.double().cpu().numpy() for x in cache.rows(held, int(held.max())))
        for b, row in enumerate(oracle):
            for h, o in enumerate(row):
                n = len(o)
                assert np.array_equal(ks[b, h, :n], o.k) and np.array_equal(vs[b, h, :n], o.v) and ids[b, h, :n].tolist() == o.ids
                ref, p, spread, _ = o.attend(_f64(qn[b, h * 4:h * 4 + 4]))
                assert np.all(np.abs(_f64(got[b, h * 4:h * 4 + 4]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * spread + 1e-6)
                assert np.allclose(_f64(cache.weights[b, h, :n]), _f64(before[b, h, :n]) + p.sum(0), rtol=1e-5, atol=1e-7)
        assert int(cache.status) == 0


# --------------------------------------------------------------------------------------------------------- refusals
INVALID, UNSUPPORTED = 1, 7


def _desc(**kw):
    base = dict(num_seqs=2, total=100, num_heads=4, num_kv_heads=2, head_dim=128, dtype=1, **{
        f"{t}_{n}_stride": s for t, (a, b) in dict(q=(512, 128), k=(256, 128), v=(256, 128), out=(512, 128)).items()
        for n, s in (("token", a), ("head", b))})
    base.update(kw)
    return B.PackedDesc(*[base[n] for n, _ in B.PackedDesc._fields_])


@pytest.mark.parametrize("kw,code", [(dict(num_seqs=-1), INVALID), (dict(total=-1), INVALID), (dict(num_heads=3), INVALID),
                                     (dict(num_kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED),
                                     (dict(q_token_stride=500), INVALID), (dict(k_head_stride=0), INVALID),
                                     (dict(k_token_stride=-256), INVALID), (dict(total=2 ** 31 - 1), UNSUPPORTED),
                                     (dict(total=2 ** 30, num_heads=512), UNSUPPORTED)])
def test_shapes_are_checked_without_a_gpu(kw, code):
    build()
    lib, d = B.load(), _desc(**kw)
    assert lib.st3_packed_attend(C.byref(d), 4096, 4096, 4096, 4096, 4096, None, None, None) == code
    assert lib.st3_packed_weights(C.byref(d), 4096, 4096, 4096, 4096, 4096, 128, 0, None, None) == code


def test_pointers_are_checked_without_a_gpu():
    build()
    lib = B.load()

    def attend(d=None, q=4096, k=4096, v=4096, cu=4096, out=4096, lse=None):
        return lib.st3_packed_attend(C.byref(d or _desc()), q, k, v, cu, out, lse, None, None)

    assert lib.st3_packed_attend(None, 4096, 4096, 4096, 4096, 4096, None, None, None) == INVALID
    assert attend(q=None) == INVALID and attend(k=4104) == INVALID and attend(v=None) == INVALID and attend(out=4100) == INVALID
    assert attend(cu=None) == INVALID and attend(lse=2) == INVALID
    assert attend(_desc(v_head_stride=4)) == INVALID and attend(_desc(out_token_stride=0)) == INVALID
    assert attend(_desc(total=0)) == 0 and attend(_desc(num_seqs=0)) == 0

    def weights(capacity=128, window=0, lse=4096, w=4096, d=None):
        return lib.st3_packed_weights(C.byref(d or _desc()), 4096, 4096, lse, 4096, w, capacity, window, None, None)

    assert weights(capacity=0) == INVALID and weights(window=-1) == INVALID and weights(lse=None) == INVALID and weights(w=None) == INVALID
    assert weights(d=_desc(total=0)) == 0


@gpu
def test_tensors_of_the_wrong_kind_are_refused():
    q, k, v = _inputs([10], 4, 2, 64, layout="dense")
    cu, out, lse = _starts([10]), torch.empty_like(q), torch.empty(4, 10, device="cuda")
    bad = [lambda: B.packed_attend(q, k[:5], v, cu, out, lse), lambda: B.packed_attend(q, k, v[:, :1], cu, out, lse),
           lambda: B.packed_attend(q, k, v, cu.long(), out, lse), lambda: B.packed_attend(q, k, v, cu, out.float(), lse),
           lambda: B.packed_attend(q, k, v, cu, out, lse.t()), lambda: B.packed_attend(q, k, v.cpu(), cu, out, lse),
           lambda: B.packed_weights(q, k, lse, cu, torch.zeros(2, 2, 64, device="cuda")),
           lambda: B.packed_weights(q, k, lse[:2], cu, torch.zeros(1, 2, 64, device="cuda"))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(B.St3Error):
        B.packed_attend(q.float(), k.float(), v.float(), cu, out.float(), lse)


@gpu
@pytest.mark.parametrize("lens,heads,kv,dim,window", [
    ([700], 32, 8, 128, 0), ([700], 4, 1, 64, 0), ([1300], 6, 2, 64, 0), ([257], 3, 3, 64, 0), ([1], 16, 1, 128, 0), ([130], 16, 1, 64, 1),
    ([2000, 3], 2, 1, 64, 900), ([500, 0, 700], 8, 4, 64, 0), ([1500], 8, 1, 128, 200)])
def test_weights_of_few_items_are_shared_by_blocks(lens, heads, kv, dim, window):
    """A prompt or two: the steps of an item go to 2, 4 or 8 blocks, whose sums are joined in one order."""
    q, k, v = _inputs(lens, heads, kv, dim, seed=3)
    lse = _attend(q, k, v, lens)[1]
    cap = -(-max(lens) // 64) * 64
    w = torch.full((len(lens), kv, cap), -1.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.packed_weights(q, k, lse, _starts(lens), w, window, status)
    again = torch.full_like(w, -1.0)
    B.packed_weights(q, k, lse, _starts(lens), again, window)
    assert torch.equal(w, again) and int(status) == 0
    want = O.packed_weights(_f64(q), _f64(k), _f64(lse), lens, window)
    got = w.cpu().numpy()
    for s, n in enumerate(lens):   # logits and sums below 24 together: 2^-18 * (1 + 24) < 1e-4
        assert np.allclose(got[s, :, :n], want[s], rtol=1e-4, atol=1e-30) and np.all(got[s, :, n:] == -1)
