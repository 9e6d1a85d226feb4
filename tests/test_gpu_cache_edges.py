"""The 8-bit cache where numbers run out, and calls at the edge of what the header allows."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2412_20105_b200 import binding as B
from paper_2412_20105_b200.build import build
from test_gpu_cache import INVALID, Pair, _desc, _i32, _starts

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ rows that weigh little
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [8.0, 10.0, 14.0, 16.0, 17.25, 20.0])
@pytest.mark.parametrize("noise", [0.0, 0.5])
def test_rows_behind_sinks_keep_their_share(dtype, gap, noise):
    """Rows 0, 16, 32 and 48 of every block outweigh the others by e^gap and have no value of their own: the output is what the
    others give."""
    lens, group, dim = [300, 64], 4, 64
    p = Pair(2, 2, dim, 320, dtype, seed=int(gap))
    sinks = torch.cat([torch.arange(n) % 16 == 0 for n in lens])

    def change(k, v):
        k.normal_(generator=torch.Generator().manual_seed(1)).mul_(noise)
        v.normal_(generator=torch.Generator().manual_seed(2)).add_(0.5)
        k[:, :, 0] = torch.where(sinks, gap, 0.0)[:, None].to(k.dtype)
        v[sinks] = 0

    p.store(lens, change=change)
    p.set_weights(lambda b, h, n: np.zeros(n))
    q = (torch.randn(2, 2 * group, dim, generator=torch.Generator().manual_seed(3)) * noise).to(p.rows(1).dtype)
    q[..., 0] = math.sqrt(dim)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    p.cache.attend(q.cuda(), _i32(lens), out)
    assert int(p.cache.status) == 0
    for b in range(2):
        for h in range(2):
            o = p.o[b][h]
            n = len(o)
            ref, prob, spread, reach = o.attend(q[b, h * group:(h + 1) * group].double().numpy())
            got = out[b, h * group:(h + 1) * group].double().cpu().numpy()
            # Logits, exp2 and the output's rounding as in Pair.attend.  A probability times its block's scale is held relative to
            # 2^-15 of the largest so far, in f16 (10 bits behind the first: half a step is 2^-11 of one term; in fp32 a second term
            # takes the rest, 2^-22) with an absolute half step of 2^-25 below 2^-14, that is 2^-40 of the largest, which meets
            # codes of up to 127.
            logit = 2.0 ** -20 * reach + 2.0 ** -20
            half, step = (2.0 ** -8, 2.0 ** -11) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -22)
            largest = (prob * np.repeat(o.vs, 64)[:n]).max() * 127
            bound = half * np.abs(ref) + (step + 2 * logit) * spread + n * 2.0 ** -40 * largest + 1e-30
            assert np.all(np.abs(got - ref) <= bound), (b, h, float((np.abs(got - ref) / bound).max()))


# --------------------------------------------------------------------------------------------------- calls at the edge
def test_a_target_on_another_device_is_refused():
    """Ahead of any launch: stand-ins, as there may be one GPU or none."""
    class Other:
        _index, desc = 1, _desc()

    cache = object.__new__(B.Cache)
    cache._index, cache.desc, cache.torch, cache.batch, cache._workspaces = 0, _desc(), torch, 2, {}
    counts = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="cuda:1"):
        cache.evict(counts, counts, 8, into=Other())


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses stand in for tensors")
def test_strides_of_one_head_may_be_anything():
    """Without a GPU the call gets as far as the launch."""
    build()
    lib, d = B.load(), _desc(num_kv_heads=1)

    def store(kt=128, kh=128, vt=128, vh=128, total=5):
        return lib.st3_cache_store(C.byref(d), 4096, 4096, 1, kt, kh, vt, vh, 4096, total, None, None, None, None)

    assert store(kh=-3, vh=1) != INVALID and store(kt=-1, vt=5, total=1) != INVALID
    assert store(kt=4) == INVALID and store(vt=-128) == INVALID


@gpu
def test_one_head_or_one_row_with_strides_of_any_kind():
    odd = lambda x, token, head: x.as_strided(x.shape, (x.stride(0) if token is None else token, x.stride(1) if head is None else head, 1))
    for heads, n in ((1, 90), (2, 1)):
        p, other = Pair(1, heads, 64, 128), B.Cache.empty(1, heads, 64, 128)
        p.store([n])
        k, v, _, _ = p.cache.rows(_i32([n]), n)
        k, v = (x[0].transpose(0, 1).contiguous() for x in (k, v))
        if heads == 1:
            k, v = odd(k, None, 7), odd(v, None, 1)
        else:
            k, v = odd(k, 3, None), odd(v, 0, None)
        other.store(k, v, _starts([n]))
        p.check(other, weights=False)


@gpu
@pytest.mark.parametrize("cu,start", [([0, 640, 0, 640], None), ([0, 64, 0, 64], None), ([0, 640, 639, 640], None), ([640, 0, 0, 0], None),
                                      ([0, 640, 640, 641], None), ([0, 10, 20, 30], [0, 0, 700]), ([0, 0, 0, 10], [0, 700, 0])])
def test_every_kind_of_wrong_offsets_is_reported(cu, start):
    """Also where no block falls to the sequence that is wrong, and where a sequence without rows starts beyond the cache."""
    p = Pair(3, 2, 64, 640)
    k = torch.randn(640, 2, 64, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    p.cache.store(k, k, _i32(cu), start=None if start is None else _i32(start))
    empty_beyond = start == [0, 700, 0]
    assert int(p.cache.status) == (0 if empty_beyond else B.DEV_RANGE)


def test_streams_are_found_without_what_torch_may_not_offer(monkeypatch):
    class Stream:
        cuda_stream = 1234

    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.delattr(torch._C, "_cuda_getDevice", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: Stream if index == 3 else None)
    assert B._stream_of(3) == 1234
    with pytest.raises(ValueError, match="cuda:2"):
        B._stream_of(2)


def test_numbers_beyond_32_bits_are_refused_not_cut():
    """ctypes would cut 2^32 + 5 to 5."""
    cache = object.__new__(B.Cache)
    cache._index, cache.desc, cache.torch, cache.batch, cache.status = 0, _desc(), torch, 2, torch.zeros(1, dtype=torch.int32)
    counts = torch.zeros(2, dtype=torch.int32)
    for keep, recent in ((2 ** 32 + 5, 0), (2 ** 31, 1), (8, 2 ** 32), (-2 ** 32 + 8, 0)):
        with pytest.raises(ValueError, match="32 bits"):
            cache.evict(counts, counts, keep, recent)


@gpu
def test_a_window_beyond_32_bits_is_refused():
    build()
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(1, 1, 64, device="cuda")
    for window in (2 ** 31, 2 ** 32, 2 ** 32 + 3, -2 ** 32 + 1):
        with pytest.raises(ValueError, match="32 bits"):
            B.packed_weights(q, k, torch.zeros(2, 4, device="cuda"), _starts([4]), w, window)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [128, 130, 260])
def test_groups_beyond_a_pass_of_the_joining_launch(group, dtype):
    p = Pair(2, 1, 64, 200, dtype, seed=group)
    p.store([150, 7])
    p.set_weights(lambda b, h, n: p.g.exponential(size=n))
    p.attend(group)
