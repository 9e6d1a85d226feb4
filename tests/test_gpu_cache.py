"""The 8-bit cache of grouped heads through the C ABI against its fp64 oracle."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2412_20105_b200 import binding as B
from paper_2412_20105_b200.build import build

gpu = pytest.mark.gpu
_T = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(lens):
    return _i32([0] + list(np.cumsum(lens)))


class Pair:
    """A cache on the GPU and its oracle, fed the same rows."""

    def __init__(self, batch, heads, dim, cap, dtype="bf16", seed=0):
        build()
        self.g = np.random.default_rng(seed)
        self.dtype, self.dim, self.batch, self.heads = dtype, dim, batch, heads
        self.cache = B.Cache.empty(batch, heads, dim, cap)
        for x in (self.cache.k, self.cache.v):      # whatever an earlier use has left
            x.random_(-128, 128)
        for x in (self.cache.k_scale, self.cache.v_scale, self.cache.weights):
            x.fill_(float("nan"))
        self.cache.ids.fill_(-7)
        self.o = [[O.Head(dim) for _ in range(heads)] for _ in range(batch)]
        self.seen = [0] * batch

    def held(self):
        return [len(h[0]) for h in self.o]

    def rows(self, n, size=1.0):
        x = self.g.normal(size=(n, self.heads, self.dim)) * size
        x *= 2.0 ** self.g.integers(-3, 4, size=(1, self.heads, self.dim))
        return torch.tensor(x, dtype=torch.float32).to(_T[self.dtype])

    def store(self, lens, size=1.0, change=None, strided=False):
        k, v = self.rows(sum(lens), size), self.rows(sum(lens), size)
        if change:
            change(k, v)
        start, pos, lo = self.held(), list(self.seen), 0
        for b, n in enumerate(lens):
            for h in range(self.heads):
                self.o[b][h].store(k[lo:lo + n, h].double().numpy(), v[lo:lo + n, h].double().numpy(), pos[b])
            self.seen[b] += n
            lo += n
        kg, vg = k.cuda(), v.cuda()
        if strided:    # slices of one tensor, and heads ahead of tokens
            kg = torch.cat([kg, kg], 1)[:, self.heads:]
            vg = vg.transpose(0, 1).contiguous().transpose(0, 1)
        self.cache.store(kg, vg, _starts(lens), start=_i32(start), pos=_i32(pos))

    def check(self, cache=None, weights=True):
        cache = cache or self.cache
        held = self.held()
        n = max(held) + 3
        k, v, ids, w = (x.cpu() for x in cache.rows(_i32(held), n, dtype=torch.float32))
        k16, v16, _, _ = cache.rows(_i32(held), n)
        assert torch.equal(k16.float().cpu(), k) and torch.equal(v16.float().cpu(), v)     # values are exact in bf16
        for b in range(self.batch):
            for h in range(self.heads):
                o = self.o[b][h]
                m = len(o)
                assert np.array_equal(k[b, h, :m].double().numpy(), o.k), (b, h)
                assert np.array_equal(v[b, h, :m].double().numpy(), o.v), (b, h)
                assert ids[b, h, :m].tolist() == [int(i) for i in o.ids]
                if weights:
                    assert np.array_equal(w[b, h, :m].double().numpy(), np.array(o.weights), equal_nan=True)
                assert not k[b, h, m:].any() and not v[b, h, m:].any() and not ids[b, h, m:].any()
        assert int(cache.status) == 0

    def set_weights(self, f):
        """f(b, h, n) -> the weights of a head, in the cache and in the oracle."""
        for b in range(self.batch):
            for h in range(self.heads):
                o = self.o[b][h]
                w = np.asarray(f(b, h, len(o)), dtype=np.float32)
                o.weights = [float(x) for x in w]
                self.cache.weights[b, h, :len(o)] = torch.from_numpy(w).cuda()

    def attend(self, group, accumulate=True, seed=1, q=None):
        if q is None:
            q = torch.randn(self.batch, self.heads * group, self.dim, generator=torch.Generator().manual_seed(seed)).to(_T[self.dtype]) * 1.5
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        before = self.cache.weights.clone()
        self.cache.attend(q.cuda(), _i32(self.held()), out, weights_out=self.cache.weights if accumulate else None)
        assert int(self.cache.status) == 0
        after = self.cache.weights.cpu()
        for b in range(self.batch):
            for h in range(self.heads):
                o = self.o[b][h]
                n = len(o)
                ref, p, spread, reach = o.attend(q[b, h * group:(h + 1) * group].double().numpy())
                got = out[b, h * group:(h + 1) * group].double().cpu().numpy()
                # Logits: exact products, fp32 sums of D terms in 16s and a handful of fp32 operations: 2^-20 of the largest sum of
                # magnitudes.  Probabilities: f16 (half a step of 11 bits; at fp32 two terms, 2^-21) with an absolute step
                # of 2^-24 of the largest (probability * scale), which meets codes of up to 127; exp2 and sums 2^-20; the
                # output's own rounding.
                logit = 2.0 ** -20 * reach + 2.0 ** -20
                half, step = (2.0 ** -8, 2.0 ** -11) if self.dtype == "bf16" else (2.0 ** -24, 2.0 ** -21)
                largest = (p * np.repeat(o.vs, 64)[:n]).max() * 127 if n else 0.0
                bound = half * np.abs(ref) + (step + 2 * logit) * spread + (n * 2.0 ** -24 * largest + 1e-30)
                assert np.all(np.abs(got - ref) <= bound), (b, h, n, float((np.abs(got - ref) - bound).max()))
                if accumulate:
                    was = before[b, h, :n].double().cpu().numpy()
                    want = was + p.sum(0)
                    tol = 2 * logit * p.sum(0) + 2.0 ** -23 * np.abs(want) + 1e-30
                    assert np.all(np.abs(after[b, h, :n].double().numpy() - want) <= tol), (b, h)
                    o.weights = [float(x) for x in after[b, h, :n]]
                    rest = (after[b, h, n:], before[b, h, n:].cpu())
                    assert torch.equal(rest[0].view(torch.int32), rest[1].view(torch.int32))       # left as they were
        if not accumulate:
            assert torch.equal(after.view(torch.int32), before.cpu().view(torch.int32))
        return out

    def evict(self, keep, recent, into=None):
        held = _i32(self.held())
        new = self.cache.evict(held, _i32(self.seen), keep, recent, into=into)
        for row in self.o:
            for o in row:
                o.evict(keep, recent, self.seen[self.o.index(row)])
        assert new.tolist() == self.held()
        return new


# --------------------------------------------------------------------------------------------------------- rows in
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_then_pieces_then_single_tokens(dtype, dim):
    p = Pair(3, 2, dim, 320, dtype)
    p.store([1, 64, 130])
    p.check()
    p.store([62, 1, 0], size=0.1)
    p.check()
    p.store([1, 1, 1], size=30.0)          # the blocks' scales grow
    p.check()
    p.store([1, 66, 63], size=4.0, strided=True)
    p.check()
    p.store([0, 0, 1])
    p.check()


@gpu
def test_values_at_the_borders_of_scales_and_codes():
    p = Pair(1, 1, 64, 128, "f32")

    def change(k, v):
        k.zero_()
        v.zero_()
        k[0, 0, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, 126.5])             # ties, the largest code
        v[0, 0, :4] = torch.tensor([127.00001, 1.0, 3.0, 253.0])

    p.store([3], change=change)
    p.check()
    assert p.cache.k_scale[0, 0, 0].item() == 1.0 and p.cache.v_scale[0, 0, 0].item() == 2.0
    p.store([61], change=lambda k, v: (k.zero_(), v.mul_(1e-35)))
    p.check()
    p.store([4], change=lambda k, v: (k.mul_(1e-20), v.fill_(1e-38)))           # below and at the smallest scale
    p.check()
    p.store([1], change=lambda k, v: (k.fill_(3e38), v.fill_(-1e20)))           # beyond the largest: clamped
    p.check()
    assert p.cache.k[0, 0, 68].tolist() == [127] * 64 and p.cache.k_scale[0, 0, 1].item() == 2.0 ** 60


@gpu
def test_what_is_not_finite_is_stored_as_zero_and_reported():
    p = Pair(2, 2, 64, 64)
    p.store([2, 3], change=lambda k, v: None)
    k = p.rows(2)
    v = p.rows(2)
    k[0, 1, 3], v[1, 0, 5] = float("nan"), float("-inf")
    p.cache.store(k.cuda(), v.cuda(), _starts([1, 1]), start=_i32(p.held()))
    assert int(p.cache.status) == B.DEV_NONFINITE
    p.cache.status.zero_()
    k[0, 1, 3], v[1, 0, 5] = 0.0, 0.0
    for b in range(2):
        for h in range(2):
            p.o[b][h].store(k[b:b + 1, h].double().numpy(), v[b:b + 1, h].double().numpy())
    p.check()


@gpu
def test_rows_that_do_not_fit_are_reported_and_nothing_else_is_lost():
    p = Pair(3, 1, 64, 64)
    p.store([60, 10, 0])
    codes = p.cache.k.clone()
    k, v = p.rows(12), p.rows(12)
    p.cache.store(k.cuda(), v.cuda(), _starts([5, 4, 3]), start=_i32(p.held()))       # 65 rows in the first
    assert int(p.cache.status) == B.DEV_RANGE
    p.cache.status.zero_()
    assert torch.equal(p.cache.k[0], codes[0])
    p.o[1][0].store(k[5:9, 0].double().numpy(), v[5:9, 0].double().numpy())
    p.o[2][0].store(k[9:, 0].double().numpy(), v[9:, 0].double().numpy())
    p.check()
    for cu in ([0, 5, 4, 12], [0, 4, 13, 13], [-1, 4, 5, 6], [0, 1, 2, 13]):          # not ascending, out of the tensor
        p.cache.store(k.cuda(), v.cuda(), _i32(cu), start=_i32([64, 64, 64]))
        assert int(p.cache.status) == B.DEV_RANGE
        p.cache.status.zero_()


@gpu
def test_reading_rows_from_anywhere():
    p = Pair(2, 2, 128, 192)
    p.store([150, 40])
    k, v, ids, w = p.cache.rows(_i32([150, 40]), 70, first=_i32([100, -5]))
    for b, first in enumerate([100, -5]):
        for h in range(2):
            o = p.o[b][h]
            for i in range(70):
                r = first + i
                want = o.k[r] if 0 <= r < len(o) else np.zeros(128)
                assert np.array_equal(k[b, h, i].double().cpu().numpy(), want)
                assert int(ids[b, h, i]) == (r if 0 <= r < len(o) else 0)


# --------------------------------------------------------------------------------------------------------- attention
LENGTHS = [[1], [0, 1, 16, 17], [63, 64, 65], [1000, 0, 129, 1], [2500, 2500]]


@gpu
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("group", [1, 4, 7])
def test_attention_over_ragged_lengths(dtype, dim, lens, group):
    p = Pair(len(lens), 2, dim, max(lens) + 70, dtype, seed=len(lens) + group)
    p.store(lens)
    p.set_weights(lambda b, h, n: p.g.exponential(size=n))
    p.attend(group)
    p.attend(group, accumulate=False, seed=2)


@gpu
@pytest.mark.parametrize("group", [2, 3, 5, 8, 9, 16, 17, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_size_of_a_group(group, dtype):
    p = Pair(2, 1, 128 if group % 2 else 64, 700, dtype, seed=group)
    p.store([300, 641])
    p.set_weights(lambda b, h, n: p.g.exponential(size=n))
    p.attend(group)


@gpu
def test_many_sequences_and_more_blocks_than_the_grid():
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(0, 260, size=333)]
    p = Pair(len(lens), 2, 64, 260)
    p.store(lens)
    p.set_weights(lambda b, h, n: np.zeros(n))
    p.attend(2)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_very_different_scales(dtype):
    """V of one block is 2^40 times another's, K and q span many powers of two: one accumulator serves all blocks."""
    p = Pair(1, 1, 64, 512, dtype)
    for i, size in enumerate([1.0, 2.0 ** -30, 2.0 ** 10, 2.0 ** -12, 2.0 ** 3]):
        def change(k, v, size=size):
            k.mul_(0.1)
            v.mul_(size)
        p.store([64], change=change)
    p.set_weights(lambda b, h, n: np.zeros(n))
    p.attend(4)
    q = torch.randn(1, 4, 64).to(_T[dtype])
    q[0, 1] *= 2.0 ** -40
    q[0, 2, 1:] *= 2.0 ** -20
    q[0, 3] = 0.0
    p.attend(4, q=q)


@gpu
def test_one_token_takes_all_and_logits_far_apart():
    p = Pair(1, 1, 64, 256)

    def change(k, v):
        k.mul_(0.01)
        k[131, 0] = 100.0
    p.store([200], change=change)
    p.set_weights(lambda b, h, n: np.zeros(n))
    q = torch.ones(1, 2, 64, dtype=torch.bfloat16) * 8
    q[0, 1] *= -1
    out = p.attend(2, q=q)
    assert torch.equal(out[0, 0].double().cpu(), torch.from_numpy(p.o[0][0].v[131]))


@gpu
def test_a_query_that_is_not_finite_stays_in_its_row():
    p = Pair(1, 2, 64, 128)
    p.store([100])
    q = torch.randn(1, 4, 64, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    clean, out = torch.empty_like(q), torch.empty_like(q)
    p.cache.attend(q, _i32([100]), clean)
    q[0, 1, 7], q[0, 2, 3] = float("nan"), float("inf")
    p.cache.attend(q, _i32([100]), out)
    assert torch.equal(out[0, 0], clean[0, 0]) and torch.equal(out[0, 3], clean[0, 3])
    assert torch.isnan(out[0, 1]).all()


@gpu
def test_counts_beyond_the_capacity_are_cut_and_reported():
    p = Pair(2, 1, 64, 128)
    p.store([128, 5])
    q = torch.randn(2, 2, 64).bfloat16().cuda()
    out, ref = torch.empty_like(q), torch.empty_like(q)
    p.cache.attend(q, _i32([128, 0]), ref)
    p.cache.attend(q, _i32([1000, -3]), out)
    assert int(p.cache.status) == B.DEV_RANGE and torch.equal(out, ref) and not out[1].any()


@gpu
def test_rows_past_four_gigabytes():
    """Codes behind 2^32 bytes of the same tensor: the last sequence's rows, alone and in the batch."""
    build()
    n, heads, dim, cap = 5, 8, 128, 1 << 20
    cache = B.Cache.empty(n, heads, dim, cap)
    big = Pair(1, heads, dim, 128, seed=5)
    big.store([100])
    held = _i32([0, 0, 0, 0, 100])
    k, v, _, _ = big.cache.rows(_i32([100]), 100)
    cache.store(k[0].transpose(0, 1).contiguous(), v[0].transpose(0, 1).contiguous(), _starts([0, 0, 0, 0, 100]))
    q = torch.randn(n, heads * 2, dim, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    out, ref = torch.empty_like(q), torch.empty(1, heads * 2, dim, dtype=torch.bfloat16, device="cuda")
    cache.attend(q, held, out)
    big.cache.attend(q[4:].contiguous(), _i32([100]), ref)
    assert torch.equal(out[4], ref[0]) and not out[:4].any()
    # and at the end of a head of a million rows
    tail = cap - 128
    cache.store(k[0].transpose(0, 1).contiguous(), v[0].transpose(0, 1).contiguous(), _starts([0, 0, 0, 100, 0]),
                start=_i32([0, 0, 0, tail, 0]))
    k2, v2, ids, _ = cache.rows(_i32([0, 0, 0, tail + 100, 0]), 100, first=_i32([tail] * 5))
    assert ids[3, heads - 1].tolist() == list(range(tail, tail + 100))
    assert int(cache.status) == 0 and torch.equal(k2[3], k[0]) and torch.equal(v2[3], v[0])


# --------------------------------------------------------------------------------------------------------- eviction
@gpu
@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (63, 5), (64, 64), (65, 1), (200, 40), (500, 0)])
@pytest.mark.parametrize("out_of_place", [False, True])
def test_eviction_in_place_and_into_another_cache(keep, recent, out_of_place):
    p = Pair(3, 2, 64, 400, seed=keep)
    for size in (1.0, 0.01, 20.0):
        p.store([130, 64, 1], size=size)
    p.set_weights(lambda b, h, n: p.g.exponential(size=n))
    into = B.Cache.empty(3, 2, 64, min(keep, 512)) if out_of_place else None
    p.evict(keep, recent, into=into)
    if into is not None:
        p.cache = into
    p.check()
    if not out_of_place:                    # and on: the cache goes on being used
        p.store([1, 1, 1], size=50.0)
        p.check()
        p.attend(4)
        p.evict(max(1, keep - 1), min(recent, max(1, keep - 1)))
        p.check()


@gpu
@pytest.mark.parametrize("case", ["equal", "zeros of both signs", "infinite", "nan", "few values", "one row more"])
def test_ties_and_weights_that_are_not_ordinary(case):
    p = Pair(2, 2, 64, 512, seed=7)
    p.store([300, 301])
    p.evict(290, 0)                         # rows no longer lie in the order of their positions
    p.store([10, 11])
    rng = p.g

    def w(b, h, n):
        if case == "equal":
            return np.full(n, 0.25)
        if case == "zeros of both signs":
            return np.where(rng.random(n) < 0.5, -0.0, 0.0)
        if case == "infinite":
            return np.where(rng.random(n) < 0.5, np.inf, np.where(rng.random(n) < 0.5, -np.inf, 1.0))
        if case == "nan":
            return np.where(rng.random(n) < 0.3, np.nan, rng.exponential(size=n))
        if case == "few values":
            return rng.integers(0, 3, size=n)
        return rng.exponential(size=n)

    p.set_weights(w)
    keep = 299 if case == "one row more" else 100
    p.evict(keep, 7)
    if case == "nan":
        assert int(p.cache.status) == B.DEV_NONFINITE
        p.cache.status.zero_()
    p.check()


@gpu
@pytest.mark.parametrize("n,keep", [(2000, 700), (9500, 4000)])
@pytest.mark.parametrize("values", [1, 2, 40])
def test_more_ties_than_are_ranked_one_against_the_other(n, keep, values):
    """Thousands of rows share the weight of the cut: the earlier positions stay.  Staged in shared memory and beyond that."""
    p = Pair(1, 2, 64, n, seed=values)
    p.store([n])
    p.set_weights(lambda b, h, m: p.g.integers(0, values, size=m) * 0.5)
    p.evict(keep + n // 4, 0)               # positions no longer ascend
    p.set_weights(lambda b, h, m: p.g.integers(0, values, size=m) * -0.25)
    p.evict(keep, 50)
    p.check()


@gpu
@pytest.mark.parametrize("lens,keep,recent", [([16000, 700], 4001, 64), ([20001], 777, 0), ([39999, 10, 300, 0], 250, 250), ([70001], 30000, 5)])
@pytest.mark.parametrize("kind", ["uniform", "octaves", "few", "same", "signs"])
def test_heads_that_several_blocks_share(lens, keep, recent, kind):
    """Two, four and eight blocks to a head, and one longer than they stage; cuts among weights, among equal ones, among recent rows."""
    p = Pair(len(lens), 1, 64, -(-max(lens) // 64) * 64, seed=len(kind))
    p.store(lens)
    weights = {"uniform": lambda b, h, n: p.g.random(n), "octaves": lambda b, h, n: np.exp(p.g.uniform(-60, 60, size=n)),
               "few": lambda b, h, n: p.g.integers(0, 4, size=n) * 1.5, "same": lambda b, h, n: np.full(n, 0.25),
               "signs": lambda b, h, n: np.where(p.g.random(n) < 0.01, np.inf, p.g.normal(size=n))}[kind]
    p.set_weights(weights)
    p.evict(keep + max(lens) // 5, recent)
    p.set_weights(weights)
    p.evict(keep, recent)
    p.check()


def _scattered(n, gap, far):
    g = np.random.default_rng(n + gap)
    return np.concatenate([np.unique(g.integers(0, n * gap, size=n - 2)), [far - 1, far - 2]])


def _at_a_border(rows):
    """Positions up to 2^30 go into 2048 bins of 2^19: many rows on both sides of a border, and a bin that ends 200 short of it."""
    g, b = np.random.default_rng(rows), 5 << 19
    more = b + 300 + g.permutation((1 << 19) - 600)[:rows]
    return np.concatenate([np.arange(b - 700, b + 200), np.sort(more), [b + (1 << 19) - 201, (1 << 30) - 1]])


@gpu
@pytest.mark.parametrize("ids", [_scattered(4000, 300, 1 << 30), _scattered(20000, 50, 1 << 30), _scattered(20000, 3000, (1 << 31) - 1),
                                 _at_a_border(900), _at_a_border(9000)], ids=["4000", "20000", "far", "border", "long-border"])
def test_cuts_among_equal_weights_at_scattered_positions(ids):
    """All weights are equal, so the earliest positions stay; several histograms follow each other before the cut is found."""
    build()
    g, n, far = np.random.default_rng(1), len(ids), int(ids[-1]) + 1
    cap = -(-n // 64) * 64
    ids = g.permutation(ids).astype(np.int32)
    cache, into = B.Cache.empty(1, 1, 64, cap), B.Cache.empty(1, 1, 64, cap)
    cache.k.zero_(), cache.v.zero_(), cache.k_scale.fill_(1), cache.v_scale.fill_(1)
    cache.weights.fill_(0.125)
    cache.ids[0, 0, :n] = torch.from_numpy(ids).cuda()
    held, seen = _i32([n]), _i32([far])
    for keep in list(range(1, 40)) + list(range(690, 770)) + [int(x) for x in g.integers(40, n, size=200)]:
        left = cache.evict(held, seen, keep, into=into)
        got = into.rows(left, keep)[2][0, 0].cpu().numpy()
        want = np.concatenate([np.sort(ids[ids >= far]), np.sort(ids[ids < far])])[:keep]     # from `seen` on a row is recent
        assert int(left[0]) == keep and np.array_equal(np.sort(got), np.sort(want)), keep
    assert int(cache.status) == 0


@gpu
def test_long_heads_and_nothing_to_evict():
    p = Pair(2, 1, 64, 9000, seed=1)
    p.store([9000, 50])
    p.set_weights(lambda b, h, n: np.round(p.g.exponential(size=n), 2))
    p.evict(2500, 100)
    p.check()
    before = p.cache.k.clone()
    p.evict(2500, 100)                      # nothing changes
    assert torch.equal(before, p.cache.k)
    p.check()
    into = B.Cache.empty(2, 1, 64, 2500)
    p.evict(2500, 100, into=into)
    p.check(into)


@gpu
def test_rows_behind_the_new_length_stay_as_they_were():
    p = Pair(1, 1, 64, 256)
    p.store([200])
    p.set_weights(lambda b, h, n: p.g.exponential(size=n))
    was = [x.clone() for x in (p.cache.k, p.cache.v, p.cache.ids, p.cache.weights)]
    p.evict(90, 10)
    for x, y in zip((p.cache.k, p.cache.v, p.cache.ids, p.cache.weights), was):
        assert torch.equal(x[0, 0, 90:].view(torch.uint8), y[0, 0, 90:].view(torch.uint8))
    p.check()


# --------------------------------------------------------------------------------------------------------- streams
@gpu
def test_captured_steps_replay_and_other_streams():
    """A decode step (append, attend with accumulation, evict) captured once and replayed gives what eager calls give."""
    def build_pair():
        p = Pair(2, 2, 128, 192, seed=11)
        p.store([150, 100])
        p.set_weights(lambda b, h, n: np.linspace(0, 1, n))
        return p

    g = torch.Generator().manual_seed(3)
    steps = [[torch.randn(2, n, 128, generator=g).bfloat16().cuda() for n in (2, 2, 8)] for _ in range(4)]
    results = []
    for captured in (False, True):
        p = build_pair()
        held, seen, cu = _i32([150, 100]), _i32([150, 100]), _starts([1, 1])
        k, v, q = (x.clone() for x in steps[0])
        out = torch.empty_like(q)
        grown = torch.empty_like(held)

        def step():
            p.cache.store(k, v, cu, start=held, pos=seen)
            torch.add(held, 1, out=grown)
            seen.add_(1)
            p.cache.attend(q, grown, out, weights_out=p.cache.weights)
            p.cache.evict(grown, seen, 128, 8, held_out=held)

        outs = []
        side = torch.cuda.Stream()
        graph = None
        if captured:
            state = [x.clone() for x in (p.cache.k, p.cache.v, p.cache.k_scale, p.cache.v_scale, p.cache.ids, p.cache.weights, held, seen)]
            with torch.cuda.stream(side):
                step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for x, y in zip((p.cache.k, p.cache.v, p.cache.k_scale, p.cache.v_scale, p.cache.ids, p.cache.weights, held, seen), state):
                x.copy_(y)
        for sk, sv, sq in steps:
            k.copy_(sk), v.copy_(sv), q.copy_(sq)
            graph.replay() if captured else step()
            outs.append(out.clone())
        results.append(outs + [p.cache.weights[:, :, :100].clone(), p.cache.ids[:, :, :100].clone(), held.clone()])
        assert int(p.cache.status) == 0
    assert all(torch.equal(a, b) for a, b in zip(*results))


@gpu
def test_a_graph_keeps_its_workspace_when_other_calls_need_more():
    p = Pair(2, 2, 64, 400, seed=4)
    p.store([380, 111])
    g = torch.Generator().manual_seed(2)
    q, out = torch.randn(2, 4, 64, generator=g).bfloat16().cuda(), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    held, w = _i32([380, 111]), torch.zeros_like(p.cache.weights)
    zeros = torch.zeros_like(w)
    p.cache.attend(q, held, out, weights_out=w, weights_in=zeros)
    want, want_w = out.clone(), w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.attend(q, held, out, weights_out=w, weights_in=zeros)
    many = torch.randn(2, 64, 64, generator=g).bfloat16().cuda()
    p.cache.attend(many, held, torch.empty_like(many), weights_out=torch.empty_like(w), weights_in=zeros)
    junk = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]     # whatever was let go is taken
    out.zero_()
    graph.replay()
    assert torch.equal(out, want) and torch.equal(w, want_w) and len(junk) == 64


@gpu
def test_two_caches_on_two_streams():
    ps = [Pair(2, 4, 128, 2000, seed=s) for s in (1, 2)]
    g = torch.Generator().manual_seed(7)
    q = torch.randn(2, 16, 128, generator=g).bfloat16().cuda()
    want = []
    for p in ps:
        p.store([1999, 1500])
        out = torch.empty_like(q)
        p.cache.attend(q, _i32([1999, 1500]), out)
        want.append(out)
    held = _i32([1999, 1500])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    got = [[] for _ in ps]
    for _ in range(10):
        for p, st, outs in zip(ps, streams, got):
            with torch.cuda.stream(st):
                out = torch.empty_like(q)
                p.cache.attend(q, held, out)
                outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for outs, w in zip(got, want) for o in outs)


@gpu
def test_the_same_call_gives_the_same_bits():
    p = Pair(4, 4, 128, 1500, seed=2)
    p.store([1500, 700, 3, 1100])
    q = torch.randn(4, 16, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    got = []
    for _ in range(3):
        out, w = torch.empty_like(q), torch.zeros_like(p.cache.weights)
        p.cache.attend(q, _i32([1500, 700, 3, 1100]), out, weights_out=w, weights_in=torch.zeros_like(w))
        got.append((out, w))
    assert all(torch.equal(a, got[0][0]) and torch.equal(b, got[0][1]) for a, b in got)


# --------------------------------------------------------------------------------------------------------- refusals
def _desc(**kw):
    base = dict(batch=2, num_kv_heads=2, head_dim=128, capacity=128, k=4096, v=4096, k_scale=4096, v_scale=4096, ids=4096, weights=4096)
    base.update(kw)
    return B.CacheDesc(*[base[n] for n, _ in B.CacheDesc._fields_])


INVALID, SMALL, CAPACITY, UNSUPPORTED = 1, 2, 4, 7


@pytest.mark.parametrize("kw,code", [(dict(batch=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(capacity=0), INVALID),
                                     (dict(capacity=100), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(k=None), INVALID),
                                     (dict(v=4100), INVALID), (dict(ids=None), INVALID), (dict(weights=8), INVALID),
                                     (dict(batch=30000, num_kv_heads=64), UNSUPPORTED),
                                     (dict(batch=1024, num_kv_heads=32, capacity=1 << 17), UNSUPPORTED)])
def test_descriptors_are_checked_without_a_gpu(kw, code):
    build()
    lib, d = B.load(), _desc(**kw)
    r = C.byref(d)
    assert lib.st3_cache_store(r, 4096, 4096, 1, 256, 128, 256, 128, 4096, 5, None, None, None, None) == code
    assert lib.st3_cache_attend(r, 4096, 4096, 1, 4, 4096, None, None, 4096, 1 << 30, None, None) == code
    assert lib.st3_cache_evict(r, r, 4096, 4096, 8, 0, 4096, 4096, 1 << 30, None, None) == code
    assert lib.st3_cache_rows(r, None, 4096, 4, 4096, 4096, 1, None, None, None) == code


def test_arguments_are_checked_without_a_gpu():
    build()
    lib, d = B.load(), _desc()
    r, n = C.byref(d), C.c_size_t(0)

    def store(k=4096, dtype=1, ts=256, hs=128, cu=4096, total=5):
        return lib.st3_cache_store(r, k, 4096, dtype, ts, hs, 256, 128, cu, total, None, None, None, None)

    assert store(k=None) == INVALID and store(k=4104) == INVALID and store(dtype=5) == UNSUPPORTED
    assert store(ts=250) == INVALID and store(hs=-128) == INVALID and store(cu=None) == INVALID and store(total=-1) == INVALID
    assert store(total=0) == 0 and lib.st3_cache_store(None, 1, 1, 1, 8, 8, 8, 8, 4, 1, None, None, None, None) == INVALID

    def attend(heads=4, dtype=1, held=4096, wi=None, wo=None, ws=4096, nbytes=1 << 30, q=4096):
        return lib.st3_cache_attend(r, q, 4096, dtype, heads, held, wi, wo, ws, nbytes, None, None)

    assert attend(heads=3) == INVALID and attend(heads=0) == INVALID and attend(dtype=2) == UNSUPPORTED and attend(held=None) == INVALID
    assert attend(wo=4096) == INVALID and attend(ws=4100) == INVALID and attend(ws=None) == INVALID and attend(q=8) == INVALID
    assert attend(heads=4096) == UNSUPPORTED
    assert lib.st3_cache_attend_workspace(r, 4, 0, C.byref(n)) == 0
    plain = n.value
    assert attend(nbytes=plain - 1) == SMALL
    assert lib.st3_cache_attend_workspace(r, 4, 1, C.byref(n)) == 0 and n.value >= plain + 2 * 4 * 128 * 4
    assert lib.st3_cache_attend_workspace(r, 4, 1, None) == INVALID

    def evict(keep=8, recent=0, ws=4096, nbytes=1 << 30, to=None, held=4096):
        return lib.st3_cache_evict(r, C.byref(to) if to else r, held, 4096, keep, recent, 4096, ws, nbytes, None, None)

    assert evict(keep=0) == INVALID and evict(recent=9) == INVALID and evict(recent=-1) == INVALID and evict(held=None) == INVALID
    assert lib.st3_cache_evict_workspace(r, C.byref(n)) == 0 and evict(nbytes=n.value - 1) == SMALL and evict(ws=8) == INVALID
    other = dict(k=1 << 20, v=1 << 20, k_scale=1 << 20, v_scale=1 << 20, ids=1 << 20, weights=1 << 20)
    assert evict(to=_desc(**{**other, "num_kv_heads": 4})) == INVALID                 # another shape
    assert evict(to=_desc(**{**other, "k": 4096})) == INVALID                         # in place in part only
    assert evict(keep=100, to=_desc(**{**other, "capacity": 64})) == CAPACITY
    assert evict(keep=100, to=_desc(capacity=64)) == INVALID                          # the same arrays, another capacity
    assert lib.st3_cache_rows(r, None, None, 4, 4096, 4096, 1, None, None, None) == INVALID
    assert lib.st3_cache_rows(r, None, 4096, -1, 4096, 4096, 1, None, None, None) == INVALID
    assert lib.st3_cache_rows(r, None, 4096, 4, 4100, 4096, 1, None, None, None) == INVALID
    assert lib.st3_cache_rows(r, None, 4096, 4, 4096, 4096, 3, None, None, None) == UNSUPPORTED
    assert lib.st3_cache_rows(r, None, 4096, 0, 4096, 4096, 1, None, None, None) == 0


@gpu
def test_tensors_of_the_wrong_kind_are_refused():
    p = Pair(2, 2, 64, 128)
    k = p.rows(2).cuda()
    with pytest.raises(ValueError):
        p.cache.store(k[:, :1], k, _starts([1, 1]))
    with pytest.raises(ValueError):
        p.cache.store(k, k[:1], _starts([1, 1]))
    with pytest.raises(ValueError):
        p.cache.store(k, k, _starts([2]))
    with pytest.raises(ValueError):
        p.cache.store(k.transpose(1, 2).contiguous().transpose(1, 2), k, _starts([1, 1]))
    with pytest.raises(TypeError):
        p.cache.store(k.half(), k.half(), _starts([1, 1]))
    with pytest.raises(ValueError):
        p.cache.attend(torch.zeros(2, 4, 64, device="cuda"), _i32([1, 1]).long(), torch.zeros(2, 4, 64, device="cuda"))
    with pytest.raises(ValueError):
        p.cache.attend(torch.zeros(2, 4, 64, device="cuda"), _i32([1, 1]), torch.zeros(2, 4, 64, device="cuda").bfloat16())
    with pytest.raises(B.St3Error):
        p.cache.attend(torch.zeros(2, 3, 64, device="cuda"), _i32([1, 1]), torch.zeros(2, 3, 64, device="cuda"))
    with pytest.raises(ValueError):
        B.Cache(p.cache.k, p.cache.v, p.cache.k_scale, p.cache.v_scale[:1], p.cache.ids, p.cache.weights)
