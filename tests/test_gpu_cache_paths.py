"""The operators on a K/V cache where launches, masks, memory and values meet:
against the definitions in 64 bits with the tolerances of test_gpu_cache.py."""
import gc
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_cache as T  # noqa: E402
from test_gpu_cache import Case, S, check, ints  # noqa: E402


# ---- large values ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("t", [1, 20, 100, 200])
def test_large_values_behind_a_rising_score(dtype, d, t):
    # a slot's score is above those before it by a factor of 2^7.2 of its weight, and
    # its values are a hundredth of the largest number: no weight may exceed 1
    c = Case(dtype, d, b=1, hkv=1, g=1, cap=140, lens=(140,), t=t)
    c.q[:], c.k[:], c.kn[:] = 0, 0, 0
    c.q[..., 0] = math.sqrt(d)
    c.k[0, 0, 130, 0] = 5.0
    c.v[0, 0, 130] = 3e36 * torch.sign(c.v[0, 0, 130].float()).to(c.v.dtype)
    for x, y in ((c.dq, c.q), (c.dk, c.k), (c.dkn, c.kn), (c.dv, c.v)):
        x.copy_(y)
    T.run_attend(c)


# ---- refused appends ----------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,t", [(1, 20), (3, 20)])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("clear", [False, True])
def test_rows_of_a_refused_append_weigh_nothing(dtype, g, t, in_place, clear):
    c = Case(dtype, 64, b=3, hkv=2, g=g, cap=100, lens=(90, 40, 60), t=t, fill=0.5)
    rows, counts = np.tile(np.arange(t), (3, 1)), [t, t, t]
    rows[1, 3] = t
    tpos = np.tile(200 + np.arange(t), (3, 1))
    lse = torch.full((3, c.h, t), 3.0)
    over, bad = S().CACHE_FLAG_OVERFLOW, S().CACHE_FLAG_BAD_INDEX

    def step(rows, counts, flags):
        c.k, c.v, c.scores, c.pos, lens, want = T.append_ref(c, rows, counts, tpos)
        assert want == flags
        new = None if in_place else torch.zeros_like(c.dlen)
        c.cache.append(c.dkn, c.dvn, positions=ints(tpos), rows=ints(rows), counts=ints(counts),
                       lengths_out=new)
        if new is not None:
            c.dlen.copy_(new)
        if clear:  # the caller has seen the flags before the weights are added
            assert c.cache.flags() == flags
        c.lens = lens
        on = [0 if f else n for f, n in zip(flags, counts)]
        want, tol = T.accumulate_ref(c, lse, rows, on)
        c.cache.accumulate(c.dq, lse.cuda(), rows=ints(rows), counts=ints(counts))
        assert c.cache.flags() == ([0, 0, 0] if clear else flags)
        check("scores", c.dscores, want, tol)
        c.scores = c.dscores.cpu()

    step(rows, counts, [over, bad, 0])
    rows[1, 3] = 3
    step(rows, [5, 7, 9], [0, 0, 0])   # accepted again: weighed again
    step(rows, [t, t, t], [over, 0, over])
    step(rows, [0, 1, 2], [0, 0, 0])


# ---- the flags' memory --------------------------------------------------------

def bad_tree():
    c = Case("bf16", 64, b=2, hkv=1, g=1, cap=20, lens=(20, 7), t=6)
    return c, ints([[-1, 0, 1, 2, 3, 4], [-1, 5, 1, -7, 3, 4]])


def test_a_graph_outlives_its_cache_object():
    c, par = bad_tree()
    par.copy_(ints([[-1, 0, 1, 2, 3, 4]] * 2))
    cache, c.cache = c.cache, None
    out, lse = cache.attend(c.dq, c.dkn, c.dvn, parents=par)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(c.dq, c.dkn, c.dvn, parents=par, out=out, lse=lse)
    del cache
    gc.collect()
    others = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(3000)]
    par.copy_(ints([[-1, 0, 1, 2, 3, 4], [-1, 5, 1, -7, 3, 4]]))
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
    assert not any(x.any() for x in others)


def busy(seconds=0.05):
    """Work on the current stream for a while."""
    x = torch.ones(4096, 4096, device="cuda")
    for _ in range(int(seconds * 1000)):
        x @ x


def test_first_call_on_a_stream_that_does_not_wait():
    c, par = bad_tree()
    s = torch.cuda.Stream()
    busy(0.001)
    torch.cuda.synchronize()
    busy()
    cache = S().KVCache(c.dk, c.dv, c.dlen)
    cache.attend(c.dq, c.dkn, c.dvn, parents=par, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert cache.flags() == [0, S().CACHE_FLAG_BAD_INDEX]


def test_a_cache_object_dropped_before_its_call_ends():
    c, par = bad_tree()
    s = torch.cuda.Stream()
    torch.zeros(2, dtype=torch.int32, device="cuda").any()
    cache = S().KVCache(c.dk, c.dv, c.dlen)
    with torch.cuda.stream(s):
        busy(0.001)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        busy(0.3)
    cache.attend(c.dq, c.dkn, c.dvn, parents=par, stream=s)
    del cache
    gc.collect()
    others = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(500)]
    torch.cuda.synchronize()
    assert not any(x.any() for x in others)


# ---- long lists ---------------------------------------------------------------

@pytest.mark.parametrize("in_place", [True, False])
def test_append_with_a_long_list_of_few_rows(in_place):
    # as many 16-byte pieces as a launch's threads would be counted in 33 bits
    c = Case("f32", 128, b=1, hkv=1, g=1, cap=40, lens=(30,), t=4)
    n = (1 << 27) + 5
    rows = torch.full((1, n), 99, dtype=torch.int32, device="cuda")  # behind the count: not looked at
    rows[0, :3] = ints([2, 0, 3])
    tpos = np.arange(100, 104)[None]
    k, v, sc, pos, lens, flags = T.append_ref(c, np.array([[2, 0, 3]]), [3], tpos)
    new = c.dlen if in_place else torch.zeros_like(c.dlen)
    c.cache.append(c.dkn, c.dvn, positions=ints(tpos), rows=rows, counts=ints([3]),
                   lengths_out=None if in_place else new)
    torch.cuda.synchronize()
    assert new.tolist() == lens == [33] and c.cache.flags() == flags == [0]
    assert T.same(c.dk, k) and T.same(c.dv, v)
    assert torch.equal(c.dscores.cpu(), sc) and torch.equal(c.dpos.cpu(), pos)


def test_append_of_more_rows_than_blocks_in_one_go():
    # more than 2^24 pieces of 16 bytes: the blocks take turns
    n = (1 << 20) + 77
    k = torch.zeros(1, 1, n + 3, 128, device="cuda")
    v = torch.zeros_like(k)
    kn = torch.rand(1, 1, n, 128, device="cuda")
    vn = torch.rand(1, 1, n, 128, device="cuda")
    lengths = ints([2])
    S().KVCache(k, v, lengths).append(kn, vn)
    assert lengths.tolist() == [n + 2]
    assert torch.equal(k[:, :, 2:-1], kn) and torch.equal(v[:, :, 2:-1], vn)
    assert not (k[:, :, :2].any() or k[:, :, -1].any() or v[:, :, :2].any() or v[:, :, -1].any())
