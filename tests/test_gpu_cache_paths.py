"""The operators on a K/V cache where launches, masks, memory and values meet:
against the definitions in 64 bits with the tolerances of test_gpu_cache.py."""
import gc
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_cache as T  # noqa: E402
from test_gpu_cache import E32, NAN, Case, S, check, ints  # noqa: E402


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


# ---- rows of an accumulation in parts -----------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("g,t,cap,lens,counts", [
    (2, 260, 300, (300, 260, 5), (260, 100, 5)),  # 17 tiles of 32 rows: two parts
    (3, 700, 900, (900, 40), (700, 3)),           # 66: eight parts, more than the 9 rows of an entry have tiles
    (1, 1000, 1300, (1300, 0, 1029), (999, 0, 1000)),
    (5, 512, 520, (513,), (512,)),
])
def test_accumulate_in_row_parts(dtype, d, g, t, cap, lens, counts):
    c, c2 = (Case(dtype, d, b=len(lens), hkv=1, g=g, cap=cap, lens=lens, t=t, seed=t) for _ in range(2))
    rows = np.random.default_rng(t).permuted(np.tile(np.arange(t), (len(lens), 1)), axis=1)
    lse = T.real_lse(c, rows, counts)
    T.run_accumulate(c, rows=rows, counts=counts, lse=lse)
    c2.cache.accumulate(c2.dq, lse.cuda(), rows=ints(rows), counts=ints(counts))
    assert torch.equal(c.dscores, c2.dscores)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accumulate_in_row_parts_sees_all(dtype):
    c = Case(dtype, 64, b=2, hkv=2, g=1, cap=700, lens=(700, 301), t=530)
    T.run_accumulate(c, causal=False, counts=[530, 211])


def test_accumulate_over_many_slots_in_row_parts():
    # more blocks of slots and parts than the chip holds at once
    c, c2 = (Case("bf16", 64, b=1, hkv=2, g=8, cap=80000, lens=(79990,), t=130, scores=True) for _ in range(2))
    # 1,040 rows of a head; the reference for all heads at once
    q = c.q[0].double().cuda() / 8.0
    k = c.k[0, :, :79990].double().cuda()
    see = torch.arange(79990, device="cuda")[None] < 79990 - 130 + 1 + torch.arange(130, device="cuda")[:, None]
    lse = torch.empty(1, c.h, 130)
    want = c.scores.double()[0, :, :79990].cuda()
    tol = torch.zeros_like(want)
    for h in range(c.h):
        s = (q[h] @ k[h // 8].T).masked_fill_(~see, -math.inf)
        lse[0, h] = torch.logsumexp(s, 1).float()
        z = lse[0, h].double().cuda()[:, None]
        p = torch.exp(s - z)
        want[h // 8] += p.sum(0)
        # |s| is at most sum |q_i k_i|
        a = q[h].abs() @ k[h // 8].abs().T
        tol[h // 8] += (p * ((c.d + 4) * E32 * a + 4 * E32 * (1 + a + z.abs()) + (130 * 8 + 2) * E32)).sum(0)
    tol += 2 * E32 * want.abs()
    for x in (c, c2):
        x.cache.accumulate(x.dq, lse.cuda())
    check("scores", c.dscores[0, :, :79990], want.cpu(), tol.cpu().numpy())
    assert torch.equal(c.dscores, c2.dscores)


# ---- attention in parts -------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("b,hkv,g,t,cap,lens,counts", [
    (1, 1, 1, 2701, 300, (290,), None),                       # more than 2,560 rows, few parts: joined
    (2, 2, 1, 1290, 700, (700, 33), (1290, 1285)),            # by a group of lanes a row
    (1, 2, 3, 451, 2000, (1999,), (447,)),
])
def test_many_rows_in_parts(dtype, d, b, hkv, g, t, cap, lens, counts):
    run_attend_many(Case(dtype, d, b=b, hkv=hkv, g=g, cap=cap, lens=lens, t=t), counts)


def run_attend_many(c, counts):
    """T.run_attend for many rows of a chain: the reference a head at a time."""
    m = [c.t] * c.b if counts is None else list(counts)
    out0 = torch.full(c.q.shape, 7.0, dtype=T.tdt(c.dtype))
    lse0 = torch.full((c.b, c.h, c.t), -5.0)
    out, lse = out0.cuda(), lse0.cuda()
    c.cache.attend(c.dq, c.dkn, c.dvn, counts=None if counts is None else ints(counts), out=out, lse=lse)
    torch.cuda.synchronize()
    ref, zref = out0.double(), lse0.double()
    tout, tlse = torch.zeros_like(ref), torch.zeros_like(zref)
    u = 2.0 ** -8 if c.dtype == "bf16" else 0.0
    uo = 2.0 ** -8 if c.dtype == "bf16" else E32
    for b in range(c.b):
        n, w = c.lens[b], m[b]
        see = torch.ones(w, n + w, dtype=torch.bool).tril(n).cuda()
        for h in range(c.h):
            j = h // c.g
            q = c.q[b, h, :w].double().cuda() / math.sqrt(c.d)
            k = torch.cat([c.k[b, j, :n], c.kn[b, j, :w]]).double().cuda()
            v = torch.cat([c.v[b, j, :n], c.vn[b, j, :w]]).double().cuda()
            s = (q @ k.T).masked_fill_(~see, -math.inf)
            z = torch.logsumexp(s, 1)
            p = torch.exp(s - z[:, None])
            o, a = p @ v, p @ v.abs()
            most = (q.abs() @ k.abs().T).masked_fill_(~see, 0)  # at least |s|
            ds = ((c.d + 4) * E32 * most + 4 * E32 * (1 + most + z.abs()[:, None])).amax(1) + see.sum(1) * E32
            e = a * (u + 2 * ds[:, None])
            ref[b, h, :w], zref[b, h, :w] = o.cpu(), z.cpu()
            tout[b, h, :w] = (e + uo * (o.abs() + e) + 1e-30).cpu()
            tlse[b, h, :w] = (ds + E32 * 4 * (1 + z.abs())).cpu()
    check("out", out, ref, tout.numpy())
    check("lse", lse, zref, tlse.numpy())


# rows of a head: 30 and 63 (one set of 32 rows a block in bf16), 120 and 300 (two), 250 (four)
ROWS = [(1, 30), (3, 21), (1, 120), (2, 150), (1, 250)]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("mask", ["full", "tree"])
def test_masks_over_parts(dtype, d, g, t, mask):
    # a part is a step or two here, so that the new tokens' tiles are parts of their own
    c = Case(dtype, d, b=3, hkv=1, g=g, cap=1500, lens=(1500, 0, 77), t=t, seed=t)
    counts = [t, t - 1, t // 2]
    for i, n in enumerate(counts):  # never used
        c.dkn[i, :, n:] = NAN
        c.dvn[i, :, n:] = NAN
    T.run_attend(c, parents=T.some_parents(3, t, t) if mask == "tree" else None, counts=counts,
                 causal=mask != "full")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,t", ROWS)
@pytest.mark.parametrize("mask", ["causal", "full", "tree"])
@pytest.mark.parametrize("value", [NAN, math.inf, -math.inf])
def test_values_that_are_not_finite_over_parts(dtype, g, t, mask, value):
    # in a whole tile, in the last slots and in new tokens, each in a channel of its
    # own: they reach the rows that see them, whichever part they were in
    c = Case(dtype, 64, b=1, hkv=1, g=g, cap=1200, lens=(1195,), t=t, seed=t)
    par = T.some_parents(1, t, 9)
    for x, y in ((c.v, c.dv), (c.vn, c.dvn)):
        if x is c.v:
            x[0, 0, 300, 3] = value
            x[0, 0, 1194, 9] = value
        else:
            x[0, 0, t // 2, 20] = value
            x[0, 0, t - 1, 40] = value
        y.copy_(x)
    T.run_attend(c, parents=par if mask == "tree" else None, causal=mask != "full")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,t", ROWS)
def test_new_key_that_is_nan_over_parts(dtype, g, t):
    c = Case(dtype, 128, b=1, hkv=1, g=g, cap=1200, lens=(1195,), t=t, seed=t)
    c.kn[0, 0, t // 2, 3] = NAN
    c.dkn.copy_(c.kn)
    T.run_attend(c, parents=T.some_parents(1, t, 4))


@pytest.mark.parametrize("layout", ["bnhd", "padded"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts_over_parts(dtype, layout):
    for d, g, t in ((64, 2, 9), (128, 1, 110), (64, 1, 240)):
        T.run_attend(Case(dtype, d, b=2, hkv=2, g=g, cap=900, lens=(900, 350), t=t, layout=layout))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_repeats_itself(dtype):
    c = Case(dtype, 128, b=3, hkv=2, g=3, cap=5000, lens=(5000, 17, 2222), t=70)
    first = c.cache.attend(c.dq, c.dkn, c.dvn)
    for _ in range(5):
        again = c.cache.attend(c.dq, c.dkn, c.dvn)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- graphs over growing and shrinking caches ----------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,t", [(2, 300), (1, 9), (4, 20)])
def test_a_graph_cuts_its_parts_anew(dtype, g, t):
    # captured once, replayed at other lengths and counts: the same as eager calls, bit for bit
    cap, budget = 26000, 25000
    c = Case(dtype, 64, b=2, hkv=1, g=g, cap=cap, lens=(cap, cap), t=t, fill=0.5)
    state = (c.dk, c.dv, c.dscores, c.dpos, c.dlen)
    start = [x.clone() for x in state]
    out, lse = torch.zeros_like(c.dq), torch.zeros(2, c.h, t, device="cuda")
    counts, tpos = ints([0, 0]), ints(np.tile(30000 + np.arange(t), (2, 1)))

    def step():
        c.cache.attend(c.dq, c.dkn, c.dvn, counts=counts, out=out, lse=lse)
        c.cache.append(c.dkn, c.dvn, positions=tpos, counts=counts)
        c.cache.accumulate(c.dq, lse, counts=counts)
        c.cache.evict(budget, n_sink=10, n_recent=500)

    def begin(lens, n):
        for x, y in zip(state, start):
            x.copy_(y)
        c.dlen.copy_(ints(lens))
        counts.copy_(ints(n))
        out.zero_(), lse.zero_()

    begin((100, 200), (t, t))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens, n in (((cap - t, 0), (t, t)), ((3, 25500), (t, t // 2)), ((0, 0), (1, t)),
                    ((12345, 24990), (0, t)), ((cap, 700), (t, t)), ((25001, 25000), (1, 1))):
        begin(lens, n)
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (*state, out, lse)]
        flags = c.cache.flags()
        begin(lens, n)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*state, out, lse), want):
            assert torch.equal(x, y)
        assert c.cache.flags() == flags


# ---- evictions of very large caches ---------------------------------------------

@pytest.mark.parametrize("n,spread", [(300001, 0), (300001, 3000), (4194304 + 70001, 40000)])
@pytest.mark.parametrize("sink,recent", [(0, 0), (100, 20000)])
def test_evict_very_large(n, spread, sink, recent):
    # scores of which only `spread` differ: the rest are told apart by their slots, of
    # up to 23 bits; more than 1,024 blocks of 4,096 slots
    rng = np.random.default_rng(n + spread)
    score = np.full(n, 0.5, np.float32)
    score[rng.choice(n, spread, replace=False)] = rng.random(spread)
    pos = rng.permutation(n).astype(np.int32)
    k = torch.randint(-30000, 30000, (1, 1, n, 64), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    k0 = k.clone()
    dscore, dpos = torch.from_numpy(score).cuda()[None, None], torch.from_numpy(pos).cuda()[None, None]
    dscore, dpos, lengths = dscore.clone(), dpos.clone(), ints([n])
    v = torch.zeros(1, 1, n, 64, dtype=torch.bfloat16, device="cuda")
    v[0, 0, :, 0] = (torch.arange(n, device="cuda") % 251).bfloat16()
    cache = S().KVCache(k, v, lengths, scores=dscore, positions=dpos)
    for budget in (n - 777, n // 2):
        size = int(lengths[0])
        s0, p0 = dscore[0, 0, :size].cpu().numpy(), dpos[0, 0, :size].cpu().numpy()
        v0 = v[0, 0, :, 0].clone()
        k0.copy_(k)
        safe = (p0 < sink) | (p0.astype(np.int64) > int(p0.max()) - recent)
        keep = np.sort(np.lexsort((np.arange(size), -s0, ~safe))[:budget])
        src = np.arange(budget)
        free = np.ones(budget, bool)
        free[keep[keep < budget]] = False
        src[free] = keep[keep >= budget]
        cache.evict(budget, n_sink=sink, n_recent=recent)
        torch.cuda.synchronize()
        assert int(lengths[0]) == budget
        m = torch.from_numpy(src).cuda()
        assert np.array_equal(dpos[0, 0, :budget].cpu().numpy(), p0[src])
        assert np.array_equal(dscore[0, 0, :budget].cpu().numpy(), s0[src])
        assert torch.equal(v[0, 0, :budget, 0], v0[m])
        assert torch.equal(k.view(torch.int16)[0, 0, :budget], k0.view(torch.int16)[0, 0][m])


# ---- modes of the caller --------------------------------------------------------

@pytest.mark.parametrize("made,read", [(True, False), (False, True), (True, True)])
def test_flags_in_and_out_of_inference_mode(made, read):
    c, par = bad_tree()
    bad = [0, S().CACHE_FLAG_BAD_INDEX]
    with torch.inference_mode(made):
        cache = S().KVCache(c.dk, c.dv, c.dlen)
        cache.attend(c.dq, c.dkn, c.dvn, parents=par)
    with torch.inference_mode(read):
        assert cache.flags() == bad and cache.flags() == [0, 0]
        cache.attend(c.dq, c.dkn, c.dvn, parents=par)
    assert cache.flags() == bad and cache.flags() == [0, 0]


def test_library_calls_without_lse_and_flags():
    # what the header lets be NULL: the same outputs, bad indices without a flag
    import ctypes
    L, c, par = S().lib(), *bad_tree()
    ks, qs = c.dkn.stride()[:3], c.dq.stride()[:3]
    want, lse = c.cache.attend(c.dq, c.dkn, c.dvn, parents=par)
    desc = S().Cache.from_buffer_copy(c.cache.desc)
    desc.flags = None
    t = S().Tokens(1, 6, *qs, *qs, *ks, S().TOKENS_TREE)
    out = torch.zeros_like(c.dq)
    a, at = ctypes.addressof(desc), ctypes.addressof(t)
    assert L.sparsepr_cache_attend(a, at, c.dq.data_ptr(), c.dkn.data_ptr(), c.dvn.data_ptr(), par.data_ptr(),
                                   None, out.data_ptr(), None, None, 0, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # entry 0 is full, entry 1 takes its rows
    tpos = ints(np.tile(np.arange(6), (2, 1)))
    assert L.sparsepr_cache_append(a, at, c.dkn.data_ptr(), c.dvn.data_ptr(), tpos.data_ptr(), None, 6, None,
                                   c.dlen.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert c.dlen.tolist() == [20, 13]
    # without flags the caller says which entries are weighed
    before = c.dscores.clone()
    counts = ints([0, 6])
    assert L.sparsepr_cache_accumulate(a, at, c.dq.data_ptr(), lse.data_ptr(), None, 6, counts.data_ptr(), None, 0,
                                       None) == 0
    torch.cuda.synchronize()
    assert torch.equal(c.dscores[0], before[0]) and (c.dscores[1, :, :13] >= before[1, :, :13]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [3, 40])
def test_broadcast_inputs(dtype, t):
    # one query and one new key and value for all tokens, heads and entries
    c = Case(dtype, 64, b=2, hkv=2, g=2, cap=900, lens=(700, 33), t=t)
    for name, h in (("q", 4), ("kn", 2), ("vn", 2)):
        x = getattr(c, name)[:1, :1, :1].contiguous()
        setattr(c, name, x.expand(2, h, t, 64))
        setattr(c, "d" + name, x.cuda().expand(2, h, t, 64))
    see = [np.tril(np.ones((t, t), bool))] * 2
    out, lse = c.cache.attend(c.dq, c.dkn, c.dvn)
    ref, zref, tout, tlse = T.attend_ref(c, see, [t, t], torch.zeros(2, 4, t, 64), torch.zeros(2, 4, t))
    check("out", out, ref, tout)
    check("lse", lse, zref, tlse)
    tpos = np.tile(np.arange(t), (2, 1))
    k, v, sc, pos, lens, flags = T.append_ref(c, tpos, [t, t], tpos)
    c.cache.append(c.dkn, c.dvn, positions=ints(tpos))
    torch.cuda.synchronize()
    assert T.same(c.dk, k) and T.same(c.dv, v) and c.dlen.tolist() == lens
    c.k, c.v, c.scores, c.lens = k, v, sc, lens
    T.run_accumulate(c, lse=lse.cpu())
