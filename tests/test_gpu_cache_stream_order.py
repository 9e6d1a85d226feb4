"""Plain stream order for the packed prompts and the 8-bit cache: every entry point behind a producer that signals its completion
before it writes, with one set of input buffers rewritten in place from call to call and nothing synchronised between."""
import pytest
import torch

from paper_2412_20105_b200 import binding as B
from paper_2412_20105_b200.build import build
from test_gpu_stream_order import _packed

pytestmark = pytest.mark.gpu
ROUNDS = 4


def _i32(g, *values, spread=0):
    v = torch.tensor(values, dtype=torch.int32)
    return (v - (torch.randint(0, spread, v.shape, generator=g, dtype=torch.int32) if spread else 0)).cuda()


def _bf16(g, *shape):
    return torch.randn(*shape, generator=g).bfloat16().cuda()


def _packed_prompts(weights):
    def inputs(g):
        n = int(torch.randint(50, 250, (1,), generator=g))
        x = [_bf16(g, 300, 8, 128), _bf16(g, 300, 2, 128), _bf16(g, 300, 2, 128), _i32(g, 0, n, 300)]
        return x + [torch.rand(8, 300, generator=g).cuda() + 5] if weights else x

    def call(t):
        if weights:
            w = torch.zeros(2, 2, 256, device="cuda")
            B.packed_weights(t[0], t[1], t[4], t[3], w)
            return [w]
        out, lse = torch.empty_like(t[0]), torch.empty(8, 300, device="cuda")
        B.packed_attend(t[0], t[1], t[2], t[3], out, lse)
        return [out, lse]

    return inputs, call


def _cache():
    c = B.Cache.empty(2, 2, 128, 320)
    g = torch.Generator().manual_seed(0)
    c.store(_bf16(g, 600, 2, 128), _bf16(g, 600, 2, 128), _i32(g, 0, 300, 600))
    return c


def _store():
    def inputs(g):
        return [_bf16(g, 10, 2, 128), _bf16(g, 10, 2, 128), _i32(g, 0, 4, 10), _i32(g, 40, 200, spread=30)]

    def call(t):
        c = _cache()
        c.store(t[0], t[1], t[2], start=t[3])
        return list(c.rows(t[3] + 10, 320))

    return inputs, call


def _attend():
    c = _cache()

    def inputs(g):
        return [_bf16(g, 2, 8, 128), _i32(g, 300, 300, spread=250), torch.rand(2, 2, 320, generator=g).cuda()]

    def call(t):
        out, w = torch.empty_like(t[0]), torch.zeros_like(t[2])
        c.attend(t[0], t[1], out, weights_out=w, weights_in=t[2])
        return [out, w]

    return inputs, call


def _rows():
    c = _cache()

    def inputs(g):
        return [_i32(g, 300, 300, spread=250), _i32(g, 20, 20, spread=20)]

    return inputs, lambda t: list(c.rows(t[0], 100, first=t[1]))


def _evict():
    c, into = _cache(), B.Cache.empty(2, 2, 128, 64)
    weights = c.weights

    def inputs(g):
        return [torch.rand(2, 2, 320, generator=g).cuda(), _i32(g, 300, 300, spread=200), _i32(g, 300, 300, spread=3)]

    def call(t):
        c2 = B.Cache(c.k, c.v, c.k_scale, c.v_scale, c.ids, t[0])
        held = c2.evict(t[1], t[2], 64, recent=5, into=into)
        return [held] + list(into.rows(held, 64))

    return inputs, call


CALLS = {"packed_attend": lambda: _packed_prompts(False), "packed_weights": lambda: _packed_prompts(True), "store": _store,
         "attend": _attend, "rows": _rows, "evict": _evict}


@pytest.mark.parametrize("name", list(CALLS))
def test_inputs_rewritten_in_place_by_an_early_producer(name):
    import native
    build()
    lib = native.load()
    inputs, call = CALLS[name]()
    g = torch.Generator().manual_seed(len(name))
    sets = [_packed(inputs(g)) for _ in range(ROUNDS)]
    want = []
    for src, dst, views in sets:                                   # inputs in place long before the call
        dst.copy_(src)
        torch.cuda.synchronize()
        want.append([x.clone() for x in call(views)])
        torch.cuda.synchronize()
    _, dst, views = sets[0]                                        # one set of buffers for every call
    dst.zero_()
    torch.cuda.synchronize()
    got, st = [], torch.cuda.current_stream().cuda_stream
    for src, _, _ in sets:
        assert lib.st3_test_early_trigger_copy(dst.data_ptr(), src.data_ptr(), src.numel() // 16, 30, st) == 0
        got.append([x.clone() for x in call(views)])
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(want, got)):
        for j, (x, y) in enumerate(zip(a, b)):
            assert torch.equal(x, y), (name, i, j)
