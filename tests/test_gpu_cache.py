"""The operators on a K/V cache against their definitions in 64 bits on the
CPU, through the binding: attention of new tokens, append, accumulated weights,
eviction, and all four together.

Tolerances are worked out for each value from the inputs.  With e = 2^-24 (half
a step of fp32, relative) a score s = q.k / sqrt(d), summed over d products in
any order, is off by at most ds = (d + 4) e sum|q_i k_i| / sqrt(d); a weight
exp(s - lse) then by the factor ds + 4 e (1 + |s|) for the exponential and its
argument, and a sum of n of them by n e more.  bf16 adds half a step, 2^-8,
for a weight of the V product and 2^-8 for the rounded output."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E32 = 2.0 ** -24
NAN = float("nan")


def S():
    from paper_2608_18484_amd import sparsepr
    return sparsepr


def tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def ints(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


class Case:
    """Host copies (in the device's precision) and device tensors of a cache and new tokens."""

    def __init__(self, dtype="bf16", d=128, b=1, hkv=2, g=2, cap=64, lens=(40,), t=1, seed=0,
                 scale=2.0, layout="bhnd", scores=True, positions=True, fill=NAN):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.d, self.b, self.hkv, self.g, self.cap, self.t = dtype, d, b, hkv, g, cap, t
        self.h = hkv * g
        self.lens = list(lens)
        assert len(self.lens) == b
        dt = tdt(dtype)

        def mk(h, n, s=1.0):
            return (torch.randn(b, h, n, d, generator=gen) * s).to(dt)

        self.k, self.v = mk(hkv, cap), mk(hkv, cap)
        for i, n in enumerate(self.lens):  # what no slot in use holds is never used
            self.k[i, :, n:] = fill
            self.v[i, :, n:] = fill
        self.q, self.kn, self.vn = mk(self.h, t, scale), mk(hkv, t), mk(hkv, t)
        self.layout = layout
        self.dk, self.dv, self.dq, self.dkn, self.dvn = (
            self.dev(x) for x in (self.k, self.v, self.q, self.kn, self.vn))
        self.scores = torch.rand(b, hkv, cap, generator=gen)
        self.pos = torch.arange(cap, dtype=torch.int32).expand(b, hkv, cap).contiguous()
        self.dlen = ints(self.lens)
        self.dscores = self.scores.cuda() if scores else None
        self.dpos = self.pos.cuda() if positions else None
        self.cache = S().KVCache(self.dk, self.dv, self.dlen, scores=self.dscores, positions=self.dpos)

    def dev(self, x):
        """On the device in the case's layout: [B, H, N, d] itself, a view of
        [B, N, H, d], or of padded rows."""
        if self.layout == "bnhd":
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        if self.layout == "padded":
            b, h, n, d = x.shape
            y = torch.zeros(b, h, n + 3, d + 24, dtype=x.dtype)
            y[:, :, :n, :d] = x
            return y.cuda()[:, :, :n, :d]
        return x.contiguous().cuda()


def tree_mask(t, parents):
    see = np.zeros((t, t), bool)
    for u in range(t):
        w = u
        while w >= 0:
            see[u, w] = True
            w = int(parents[w])
    return see


def check(name, got, want, tol):
    """|got - want| <= tol for each value, NaN and infinities in the same places."""
    got, want = got.double().cpu().numpy(), want.numpy()
    tol = np.broadcast_to(tol, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{name}: infinities differ"
    fin = np.isfinite(want)
    assert np.isfinite(got[fin]).all(), f"{name}: not finite"
    off = np.abs(got[fin] - want[fin])
    # a tolerance of 0: the value has to be the same
    worst = float((off / np.maximum(tol[fin], 1e-300)).max()) if off.size else 0.0
    print(f"{name}: worst error {worst:.3f} of its tolerance", flush=True)
    assert worst <= 1.0, f"{name}: {worst:.2f} times its tolerance"


def attend_ref(c, see, counts, out0, lse0):
    """out, lse and their tolerances; rows behind counts as before.  `see`: per
    entry, [T, T] which token sees which."""
    out, lse = out0.double(), lse0.double()
    tout, tlse = torch.zeros_like(out), torch.zeros_like(lse)
    u = 2.0 ** -8 if c.dtype == "bf16" else 0.0
    uo = 2.0 ** -8 if c.dtype == "bf16" else E32
    for b in range(c.b):
        n, m = c.lens[b], counts[b]
        for h in range(c.h):
            j = h // c.g
            q = c.q[b, h, :m].double() / math.sqrt(c.d)
            for t in range(m):
                on = torch.from_numpy(np.flatnonzero(see[b][t, :m]))
                k = torch.cat([c.k[b, j, :n].double(), c.kn[b, j][on].double()])
                v = torch.cat([c.v[b, j, :n].double(), c.vn[b, j][on].double()])
                s = k @ q[t]
                z = torch.logsumexp(s, 0)
                p = torch.exp(s - z)
                out[b, h, t] = p @ v
                lse[b, h, t] = z
                ds = (c.d + 4) * E32 * (k.abs() @ q[t].abs()) + 4 * E32 * (1 + s.abs() + abs(z))
                w = len(s) * E32 + float(torch.nan_to_num(ds).max())
                a = p @ v.abs()
                tout[b, h, t] = a * (u + 2 * w) + uo * (out[b, h, t].abs() + a * (u + 2 * w)) + 1e-30
                tlse[b, h, t] = w + E32 * 4 * (1 + abs(z))
    return out, lse, tout.numpy(), tlse.numpy()


def run_attend(c, parents=None, counts=None, causal=True, see=None):
    m = [c.t] * c.b if counts is None else counts
    if see is None:
        if parents is not None:
            see = [tree_mask(c.t, parents[i]) for i in range(c.b)]
        elif causal:
            see = [np.tril(np.ones((c.t, c.t), bool))] * c.b
        else:
            see = [np.ones((c.t, c.t), bool)] * c.b
    out0 = torch.full(c.q.shape, 7.0, dtype=tdt(c.dtype))
    lse0 = torch.full((c.b, c.h, c.t), -5.0)
    out, lse = c.dev(out0), lse0.cuda()
    c.cache.attend(c.dq, c.dkn, c.dvn, parents=None if parents is None else ints(parents),
                   counts=None if counts is None else ints(counts), causal=causal, out=out, lse=lse)
    torch.cuda.synchronize()
    ref, zref, tout, tlse = attend_ref(c, see, m, out0, lse0)
    check("out", out, ref, tout)
    check("lse", lse, zref, tlse)
    return out, lse


def some_parents(b, t, seed=0):
    rng = np.random.default_rng(seed)
    u = np.arange(t)
    return np.maximum(u - 1 - rng.integers(0, 1 + np.minimum(u, 5), (b, t)), -1)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("length", [0, 1, 31, 32, 33, 127, 128, 129, 700])
def test_one_token(dtype, d, length):
    run_attend(Case(dtype, d, b=1, hkv=2, g=3, cap=max(length, 1), lens=(length,), t=1, seed=length))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("g,t", [(1, 1), (1, 2), (8, 1), (32, 1), (33, 1), (5, 7), (4, 16), (3, 43),
                                 (1, 31), (1, 33), (2, 70)])
def test_rows_and_ragged_lengths(dtype, d, g, t):
    run_attend(Case(dtype, d, b=3, hkv=2, g=g, cap=150, lens=(0, 150, 77), t=t, seed=g * 100 + t))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("t", [2, 29, 33, 64, 129, 256])
def test_trees(dtype, d, t):
    c = Case(dtype, d, b=2, hkv=1, g=2, cap=90, lens=(90, 3), t=t, seed=t)
    run_attend(c, parents=some_parents(2, t, t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_shapes(dtype):
    # a chain, all roots, a star and a comb, as deep and as flat as trees get
    t = 200
    u = np.arange(t)
    shapes = [u - 1, np.full(t, -1), np.where(u == 0, -1, 0), np.where(u % 2 == 0, u - 2, u - 1)]
    shapes[3][0] = -1
    c = Case(dtype, 64, b=4, hkv=1, g=1, cap=40, lens=(40, 0, 17, 33), t=t)
    run_attend(c, parents=np.stack(shapes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", ["causal", "full", "tree"])
def test_counts_leave_the_rest(dtype, mask):
    c = Case(dtype, 128, b=4, hkv=2, g=2, cap=80, lens=(80, 0, 5, 64), t=37, seed=3)
    counts = [37, 1, 0, 20]
    for i, n in enumerate(counts):  # never used
        c.dkn[i, :, n:] = NAN
        c.dvn[i, :, n:] = NAN
    run_attend(c, parents=some_parents(4, 37) if mask == "tree" else None, counts=counts,
               causal=mask != "full")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bnhd", "padded"])
def test_layouts(dtype, layout):
    run_attend(Case(dtype, 64, b=2, hkv=3, g=2, cap=101, lens=(101, 50), t=9, layout=layout))
    run_attend(Case(dtype, 128, b=2, hkv=3, g=2, cap=101, lens=(101, 50), t=70, layout=layout),
               causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [NAN, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("mask", ["causal", "tree"])
def test_bad_new_token_reaches_only_those_that_see_it(dtype, value, where, mask):
    c = Case(dtype, 64, b=1, hkv=1, g=2, cap=50, lens=(50,), t=40, seed=5)
    par = some_parents(1, 40, 9)
    see = tree_mask(40, par[0]) if mask == "tree" else np.tril(np.ones((40, 40), bool))
    bad = 10 + int(see[:, 10:30].sum(0).argmax()) if mask == "tree" else 21  # one that others continue
    if where != "v":
        c.dkn[0, 0, bad, 3] = value
    if where != "k":
        c.dvn[0, 0, bad, 5] = value
    out, lse = c.cache.attend(c.dq, c.dkn, c.dvn, parents=ints(par) if mask == "tree" else None)
    good = Case(dtype, 64, b=1, hkv=1, g=2, cap=50, lens=(50,), t=40, seed=5)
    out0 = torch.zeros(c.q.shape, dtype=tdt(dtype))
    ref, zref, tout, tlse = attend_ref(good, [see], [40], out0, torch.zeros(1, c.h, 40))
    blind = np.flatnonzero(~see[:, bad])
    assert len(blind) > 5 and see[:, bad].sum() > 1
    check("out", out[:, :, blind], ref[:, :, blind], tout[:, :, blind])
    check("lse", lse[:, :, blind], zref[:, :, blind], tlse[:, :, blind])
    if where == "v":
        seeing = torch.from_numpy(np.flatnonzero(see[:, bad])).cuda()
        col = out.float()[0][:, seeing]
        assert not torch.isfinite(col[:, :, 5]).any()
        assert torch.isfinite(torch.cat([col[:, :, :5], col[:, :, 6:]], 2)).all()
        if not math.isnan(value):
            assert (col[:, :, 5] == value).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_value_in_the_last_slot(dtype):
    # the last tile's padding repeats no row that counts
    c = Case(dtype, 64, b=1, hkv=1, g=1, cap=60, lens=(45,), t=3)
    c.dv[0, 0, 44, 7] = math.inf
    out, _ = c.cache.attend(c.dq, c.dkn, c.dvn)
    assert (out[..., 7] == math.inf).all()
    assert torch.isfinite(out[..., :7]).all() and torch.isfinite(out[..., 8:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity_and_the_lowest_value(dtype):
    low = torch.finfo(tdt(dtype)).min
    c = Case(dtype, 64, b=1, hkv=1, g=1, cap=64, lens=(64,), t=2)
    c.q[:] = c.q.abs()
    c.dq.copy_(c.q)
    # whole tiles whose scores are -inf come first and change nothing
    for i in range(40):
        c.k[0, 0, i] = -math.inf if i < 35 else low
    c.dk.copy_(c.k)
    out, lse = c.cache.attend(c.dq, c.dkn, c.dvn)
    c2 = Case(dtype, 64, b=1, hkv=1, g=1, cap=64, lens=(24,), t=2)
    c2.k[0, 0, :24], c2.v[0, 0, :24], c2.q = c.k[0, 0, 40:], c.v[0, 0, 40:], c.q
    c2.kn, c2.vn = c.kn, c.vn
    ref, zref, tout, tlse = attend_ref(c2, [np.tril(np.ones((2, 2), bool))], [2],
                                       torch.zeros(c.q.shape, dtype=tdt(dtype)), torch.zeros(1, 1, 2))
    check("out", out, ref, tout)
    check("lse", lse, zref, tlse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    # scores of a few thousand: the running maximum moves by far more than exp covers
    run_attend(Case(dtype, 128, b=2, hkv=1, g=2, cap=300, lens=(300, 11), t=5, scale=300.0))


@pytest.mark.parametrize("dtype,g,t,n,b", [("bf16", 3, 1, 20011, 2), ("bf16", 3, 21, 9001, 1),
                                           ("bf16", 2, 300, 1500, 1), ("f32", 4, 1, 6007, 2),
                                           ("f32", 2, 40, 3001, 1)])
def test_long_caches(dtype, g, t, n, b):
    # entries of very different lengths share the blocks' work
    lens = [n, n // 37][:b]
    run_attend(Case(dtype, 128, b=b, hkv=1, g=g, cap=n + 5, lens=lens, t=t))


def test_many_entries():
    lens = [int(x) for x in np.random.default_rng(2).integers(0, 60, 150)]
    run_attend(Case("bf16", 64, b=150, hkv=1, g=1, cap=60, lens=lens, t=2))


def test_bad_parents_raise_the_flag_and_count_as_roots():
    c = Case("bf16", 64, b=2, hkv=1, g=1, cap=20, lens=(20, 7), t=6)
    par = np.array([[-1, 0, 1, 2, 3, 4], [-1, 5, 1, -7, 3, 4]])
    fixed = np.array([[-1, 0, 1, 2, 3, 4], [-1, -1, 1, -1, 3, 4]])
    run_attend(c, parents=par, see=[tree_mask(6, x) for x in fixed])
    assert c.cache.flags() == [0, S().CACHE_FLAG_BAD_INDEX]
    assert c.cache.flags() == [0, 0]


def test_lengths_are_clamped_to_the_capacity():
    c = Case("bf16", 64, b=2, hkv=1, g=1, cap=20, lens=(20, 0), t=2)
    c.dlen.copy_(ints([1000, -3]))
    run_attend(c)


# ---- append -----------------------------------------------------------------

def append_ref(c, rows, counts, tpos):
    k, v, sc, pos, lens, flags = c.k.clone(), c.v.clone(), c.scores.clone(), c.pos.clone(), [], []
    for b in range(c.b):
        r = rows[b][:counts[b]]
        n = c.lens[b]
        flag = S().CACHE_FLAG_BAD_INDEX if any(x < 0 or x >= c.t for x in r) else \
            S().CACHE_FLAG_OVERFLOW if n + len(r) > c.cap else 0
        flags.append(flag)
        if flag:
            r = []
        for i, x in enumerate(r):
            k[b, :, n + i], v[b, :, n + i] = c.kn[b, :, x], c.vn[b, :, x]
            sc[b, :, n + i] = 0.0
            pos[b, :, n + i] = int(tpos[b, x])
        lens.append(n + len(r))
    return k, v, sc, pos, lens, flags


def same(a, b):
    return torch.equal(torch.nan_to_num(a.cpu().float(), nan=12345.0),
                       torch.nan_to_num(b.float(), nan=12345.0))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "padded"])
def test_append(dtype, d, listed, in_place, layout):
    t = 45
    c = Case(dtype, d, b=6, hkv=3, g=1, cap=100, lens=(0, 55, 56, 100, 99, 20), t=t, layout=layout)
    rng = np.random.default_rng(1)
    rows, counts = np.tile(np.arange(t), (6, 1)), [45, 45, 45, 0, 1, 45]
    if listed:
        rows = rng.integers(0, t, (6, t))  # the same index may come twice
        rows[5, 7] = t                     # and a bad one
        rows[0, 44] = -1                   # behind the count: not looked at
        counts[0] = 44
    tpos = rng.integers(0, 1 << 20, (6, t))
    k, v, sc, pos, lens, flags = append_ref(c, rows, counts, tpos)
    new = c.dlen if in_place else torch.full((6,), -1, dtype=torch.int32, device="cuda")
    c.cache.append(c.dkn, c.dvn, positions=ints(tpos), rows=ints(rows) if listed else None,
                   counts=ints(counts), lengths_out=None if in_place else new)
    torch.cuda.synchronize()
    assert new.tolist() == lens
    if not in_place:
        assert c.dlen.tolist() == c.lens
    assert c.cache.flags() == flags and any(flags)
    assert same(c.dk, k) and same(c.dv, v)
    assert torch.equal(c.dscores.cpu(), sc) and torch.equal(c.dpos.cpu(), pos)


def test_append_without_scores_and_positions():
    c = Case("bf16", 64, b=1, hkv=2, g=1, cap=30, lens=(7,), t=3, scores=False, positions=False)
    c.cache.append(c.dkn, c.dvn)
    assert c.dlen.tolist() == [10]
    assert torch.equal(c.dk[:, :, 7:10].cpu(), c.kn) and torch.equal(c.dv[:, :, 7:10].cpu(), c.vn)


# ---- accumulate -------------------------------------------------------------

def accumulate_ref(c, lse, rows, counts, causal=True):
    sc, tol = c.scores.double(), torch.zeros_like(c.scores).double()
    for b in range(c.b):
        n, m = c.lens[b], counts[b]
        for i, r in enumerate(rows[b][:m]):
            if r < 0 or r >= c.t:
                continue
            see = n if not causal else min(n, max(0, n - m + i + 1))
            for h in range(c.h):
                j = h // c.g
                z = float(lse[b, h, r])
                if see == 0 or z == -math.inf:
                    continue
                q = c.q[b, h, r].double() / math.sqrt(c.d)
                k = c.k[b, j, :see].double()
                s = k @ q
                p = torch.exp(s - z)
                ds = (c.d + 4) * E32 * (k.abs() @ q.abs()) + 4 * E32 * (1 + s.abs() + abs(z))
                sc[b, j, :see] += p
                tol[b, j, :see] += p * (ds + (m * c.g + 2) * E32)
        for j in range(c.hkv):
            tol[b, j, :n] += 2 * E32 * sc[b, j, :n].abs()
    return sc, tol.numpy() + 1e-30


def real_lse(c, rows, counts, causal=True):
    """The rows' log sums as attention over the slots gives them, in float32."""
    lse = torch.full((c.b, c.h, c.t), NAN)
    for b in range(c.b):
        n, m = c.lens[b], counts[b]
        for i, r in enumerate(rows[b][:m]):
            if r < 0 or r >= c.t:
                continue
            see = n if not causal else min(n, max(0, n - m + i + 1))
            for h in range(c.h):
                s = c.k[b, h // c.g, :see].double() @ c.q[b, h, r].double() / math.sqrt(c.d)
                lse[b, h, r] = float(torch.logsumexp(s, 0)) if see else -math.inf
    return lse


def run_accumulate(c, rows=None, counts=None, causal=True, lse=None):
    rr = np.tile(np.arange(c.t), (c.b, 1)) if rows is None else np.asarray(rows)
    m = [rr.shape[1]] * c.b if counts is None else counts
    lse = real_lse(c, rr, m, causal) if lse is None else lse
    want, tol = accumulate_ref(c, lse, rr, m, causal)
    c.cache.accumulate(c.dq, lse.cuda(), rows=None if rows is None else ints(rows),
                       counts=None if counts is None else ints(counts), causal=causal)
    torch.cuda.synchronize()
    check("scores", c.dscores, want, tol)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("g,t,lens", [(1, 1, (1, 0, 33)), (3, 1, (129, 32, 31)), (2, 7, (300, 7, 8)),
                                      (1, 33, (200, 33, 256)), (4, 40, (257, 90, 41)),
                                      (33, 2, (64, 65, 2))])
@pytest.mark.parametrize("causal", [True, False])
def test_accumulate(dtype, d, g, t, lens, causal):
    run_accumulate(Case(dtype, d, b=3, hkv=2, g=g, cap=300, lens=lens, t=t, seed=t), causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "padded"])
def test_accumulate_rows(dtype, layout):
    # lists with repeated and bad indices, short counts, more rows than slots
    c = Case(dtype, 64, b=4, hkv=2, g=3, cap=140, lens=(140, 20, 2, 77), t=21, layout=layout)
    rows = np.random.default_rng(4).integers(0, 21, (4, 12))
    rows[1, 3], rows[1, 4], rows[3, 11] = 21, -1, 99
    run_accumulate(c, rows=rows, counts=[12, 9, 5, 11])
    assert c.cache.flags() == [0, S().CACHE_FLAG_BAD_INDEX, 0, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accumulate_skips_empty_rows(dtype):
    c = Case(dtype, 128, b=1, hkv=1, g=2, cap=70, lens=(70,), t=3)
    rr = np.arange(3)[None]
    lse = real_lse(c, rr, [3])
    lse[0, 1, 1] = -math.inf
    run_accumulate(c, lse=lse)


def test_accumulate_long_is_repeatable():
    c = Case("bf16", 128, b=2, hkv=1, g=2, cap=9000, lens=(9000, 1234), t=150)
    c2 = Case("bf16", 128, b=2, hkv=1, g=2, cap=9000, lens=(9000, 1234), t=150)
    rows = np.tile(np.arange(150), (2, 1))
    lse = real_lse(c, rows, [150, 150])
    run_accumulate(c, lse=lse)
    c2.cache.accumulate(c2.dq, lse.cuda())
    assert torch.equal(c.dscores, c2.dscores)


def test_attention_weights_sum_to_the_rows():
    # a frame attends, enters and is weighed: every row's weights over what it saw sum to 1
    c = Case("bf16", 128, b=2, hkv=2, g=3, cap=500, lens=(430, 0), t=60)
    c.dscores.zero_()
    _, lse = c.cache.attend(c.dq, c.dkn, c.dvn)
    c.cache.append(c.dkn, c.dvn, positions=ints(np.arange(120).reshape(2, 60)))
    c.cache.accumulate(c.dq, lse)
    total = c.dscores.double().sum(2).cpu().numpy()
    # each of the 60 * 3 rows' weights: scores within 1e-4 of the attention's own
    assert np.abs(total - 180.0).max() < 180 * 2e-4


# ---- eviction ---------------------------------------------------------------

def evict_ref(lens, scores, pos, budget, n_sink, n_recent):
    """Source slot of each kept slot, per entry and K/V head."""
    src = []
    for b, n in enumerate(lens):
        per = []
        for j in range(scores.shape[1]):
            s, p = scores[b, j, :n].numpy(), pos[b, j, :n].numpy().astype(np.int64)
            if n <= budget:
                per.append(np.arange(n))
                continue
            newest = p.max()
            rank = [(2 if (n_sink + n_recent and (p[i] < n_sink or p[i] > newest - n_recent)) else
                     1 if math.isnan(s[i]) else 0, 0.0 if math.isnan(s[i]) else float(s[i]), -i)
                    for i in range(n)]
            rank = [(a, 0.0 if a == 2 else x, i) for a, x, i in rank]
            keep = sorted(-r[2] for r in sorted(rank, reverse=True)[:budget])
            late = [i for i in keep if i >= budget]
            free = np.setdiff1d(np.arange(budget), keep)
            m = np.arange(budget)
            m[free] = late
            per.append(m)
        src.append(per)
    return src


def run_evict(c, budget, n_sink=0, n_recent=0, other=None):
    src = evict_ref(c.lens, c.scores, c.pos, budget, n_sink, n_recent)
    c.dscores.copy_(c.scores)
    c.dpos.copy_(c.pos)
    k0, v0 = c.dk.clone(), c.dv.clone()
    if other:
        cap = budget + other
        to = [torch.full((c.b, c.hkv, cap, c.d), 3.0, dtype=tdt(c.dtype), device="cuda")
              for _ in range(2)]
        to += [torch.full((c.b, c.hkv, cap), 4.0, device="cuda"),
               torch.full((c.b, c.hkv, cap), 5, dtype=torch.int32, device="cuda"),
               torch.full((c.b,), -1, dtype=torch.int32, device="cuda")]
        kc = S().KVCache(to[0], to[1], to[4], scores=to[2], positions=to[3])
        c.cache.evict(budget, n_sink=n_sink, n_recent=n_recent, out=kc)
    else:
        to = [c.dk, c.dv, c.dscores, c.dpos, c.dlen]
        c.cache.evict(budget, n_sink=n_sink, n_recent=n_recent)
    torch.cuda.synchronize()
    assert to[4].tolist() == [min(n, budget) for n in c.lens]
    for b in range(c.b):
        for j in range(c.hkv):
            m = torch.from_numpy(src[b][j])
            n = len(m)
            assert same(to[0][b, j, :n], k0[b, j].cpu()[m])
            assert same(to[1][b, j, :n], v0[b, j].cpu()[m])
            assert same(to[2][b, j, :n], c.scores[b, j][m])
            assert torch.equal(to[3][b, j, :n].cpu(), c.pos[b, j][m])
            if other:  # what is behind the kept slots stays
                assert (to[0][b, j, n:] == 3).all() and (to[2][b, j, n:] == 4).all()
                assert (to[3][b, j, n:] == 5).all()
    if other:
        assert same(c.dk, k0.cpu()) and torch.equal(c.dpos.cpu(), c.pos)
        assert c.dlen.tolist() == c.lens


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("other", [0, 1, 9])
@pytest.mark.parametrize("budget,n_sink,n_recent", [(1, 0, 0), (64, 0, 0), (64, 4, 20), (64, 30, 34),
                                                    (199, 0, 1), (150, 3, 0)])
def test_evict(dtype, d, other, budget, n_sink, n_recent):
    c = Case(dtype, d, b=4, hkv=2, g=1, cap=200, lens=(200, 70, 64, 0), t=1, fill=0.5)
    run_evict(c, budget, n_sink, n_recent, other)


@pytest.mark.parametrize("kind", ["ties", "zeros", "special", "descending", "ascending"])
@pytest.mark.parametrize("n", [65, 1023, 1025, 5000])
@pytest.mark.parametrize("other", [0, 3])
def test_evict_orders(kind, n, other):
    c = Case("bf16", 64, b=1, hkv=3, g=1, cap=n, lens=(n,), t=1)
    rng = np.random.default_rng(n)
    s = c.scores.numpy()
    if kind == "ties":
        s[:] = rng.integers(0, 3, s.shape)
    elif kind == "zeros":
        s[:] = np.where(rng.random(s.shape) < 0.5, 0.0, -0.0)
    elif kind == "special":
        s[:] = rng.choice([0.0, -0.0, NAN, math.inf, -math.inf, 1e-45, -1e-45, 3e38, 1.0, -2.0], s.shape)
    elif kind == "descending":
        s[:] = -np.sort(-s, axis=2)
    else:
        s[:] = np.sort(s, axis=2)
    for budget in (n // 3, n - 1):
        run_evict(c, budget, 0, 0, other)
        c.dlen.copy_(ints(c.lens))


@pytest.mark.parametrize("kind", ["equal", "ties", "close", "special", "descending", "ascending"])
@pytest.mark.parametrize("n", [8193, 24577, 30011])
@pytest.mark.parametrize("other", [0, 3])
def test_evict_orders_of_large_caches(kind, n, other):
    # scores that only the last bits or the slots tell apart, and entries of one
    # launch that need nothing, little and much
    c = Case("bf16", 64, b=3, hkv=2, g=1, cap=n, lens=(n, n // 2 + 1, n // 3), t=1)
    rng = np.random.default_rng(n)
    s = c.scores.numpy()
    if kind == "equal":
        s[:] = 0.5
    elif kind == "ties":
        s[:] = rng.integers(0, 3, s.shape)
    elif kind == "close":  # neighbouring floats, each a few times
        s[:] = (np.float32(1.0).view(np.int32) + rng.integers(0, 1500, s.shape)).astype(np.int32).view(np.float32)
    elif kind == "special":
        s[:] = rng.choice([0.0, -0.0, NAN, math.inf, -math.inf, 1e-45, -1e-45, 3e38, 1.0, -2.0], s.shape)
    elif kind == "descending":
        s[:] = -np.sort(-s, axis=2)
    else:
        s[:] = np.sort(s, axis=2)
    for budget, sink, recent in ((n // 2, 0, 0), (n - 1, 5, 4000), (n // 3, 0, 1)):
        run_evict(c, budget, sink, recent, other)
        c.dlen.copy_(ints(c.lens))


def test_evict_goes_by_positions_not_slots():
    # after evictions the slots are not in the order of time
    c = Case("bf16", 64, b=2, hkv=2, g=1, cap=500, lens=(500, 333), t=1)
    rng = np.random.default_rng(3)
    for b in range(2):
        for j in range(2):
            c.pos[b, j] = torch.from_numpy(rng.permutation(500).astype(np.int32))
    run_evict(c, 100, 10, 50)
    # equal positions, and the largest there are
    c = Case("bf16", 64, b=1, hkv=1, g=1, cap=300, lens=(300,), t=1)
    c.pos[:] = 2 ** 31 - 1
    run_evict(c, 100, 10, 50)


@pytest.mark.parametrize("n", [33000, 70001])
def test_evict_large(n):
    c = Case("bf16", 64, b=1, hkv=2, g=1, cap=n, lens=(n,), t=1)
    run_evict(c, n - 500, 64, 3000)
    c = Case("bf16", 64, b=1, hkv=2, g=1, cap=n, lens=(n,), t=1)
    run_evict(c, n // 5, 64, 3000, other=1)


# ---- together ---------------------------------------------------------------

def rollout(dtype, steps, budget=96, t=13, seed=0, stream=None, graph=False):
    """Steps of a drafted tree's attention, the accepted path's append, its
    weights and the eviction, checked against the definitions step by step."""
    cap = budget + t
    c = Case(dtype, 64, b=2, hkv=2, g=2, cap=cap, lens=(budget, budget - 50), t=t, seed=seed, fill=0.25)
    c.dscores.zero_()
    c.scores.zero_()
    rng = np.random.default_rng(seed)
    out = torch.zeros_like(c.dq)
    lse = torch.zeros(c.b, c.h, t, device="cuda")
    par, rows, counts, tpos = ints(np.zeros((2, t))), ints(np.zeros((2, 4))), ints([0, 0]), ints(np.zeros((2, t)))

    def step(s):
        c.cache.attend(c.dq, c.dkn, c.dvn, parents=par, out=out, lse=lse, stream=s)
        c.cache.append(c.dkn, c.dvn, positions=tpos, rows=rows, counts=counts, stream=s)
        c.cache.accumulate(c.dq, lse, rows=rows, counts=counts, stream=s)
        c.cache.evict(budget, n_sink=4, n_recent=30, stream=s)

    def new_inputs(i):
        gen = torch.Generator().manual_seed(1000 * seed + i)
        for host, dev, x in ((c.q, c.dq, 2.0), (c.kn, c.dkn, 1.0), (c.vn, c.dvn, 1.0)):
            host.copy_((torch.randn(host.shape, generator=gen) * x).to(host.dtype))
            dev.copy_(host)
        p = some_parents(2, t, i)
        path = np.zeros((2, 4), int)
        n = []
        for b in range(2):
            u, way = int(rng.integers(0, t)), []
            while u >= 0:
                way.append(u)
                u = int(p[b, u])
            way = way[::-1][:4]
            n.append(len(way))
            path[b, :len(way)] = way
        # a drafted token's position is its depth's
        pos = c.next_pos[:, None] + np.stack([tree_mask(t, p[b]).sum(1) - 1 for b in range(2)])
        for dst, x in ((par, p), (rows, path), (counts, n), (tpos, pos)):
            dst.copy_(ints(x))
        c.next_pos = c.next_pos + np.asarray(n)
        return p, path, n, pos

    c.next_pos = np.asarray(c.lens)
    g = None
    if graph:
        new_inputs(99)
        n0 = [x.clone() for x in (c.dk, c.dv, c.dscores, c.dpos, c.dlen)]
        c.next_pos = np.asarray(c.lens)
        step(None)  # torch's allocator and the library are warm
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(None)
        for x, y in zip((c.dk, c.dv, c.dscores, c.dpos, c.dlen), n0):
            x.copy_(y)
    for i in range(steps):
        p, path, n, pos = new_inputs(i)
        torch.cuda.synchronize()
        if g is not None:
            g.replay()
        elif stream is not None:
            step(stream)
            stream.synchronize()
        else:
            step(None)
        torch.cuda.synchronize()
        ref, zref, tout, tlse = attend_ref(c, [tree_mask(t, p[b]) for b in range(2)], [t, t],
                                           torch.zeros(c.q.shape), torch.zeros(2, c.h, t))
        check(f"step {i} out", out, ref, tout)
        check(f"step {i} lse", lse, zref, tlse)
        k, v, sc, ps, lens, flags = append_ref(c, path, n, pos)
        assert not any(flags)
        c.k, c.v, c.scores, c.pos, c.lens = k, v, sc, ps, lens
        want, tol = accumulate_ref(c, lse.cpu(), path, n)
        # the device's own scores decide its eviction: it has to be the one that they
        # give, so near ties are taken from what it kept
        c.scores = want.float()
        margin = float(tol.max()) * (i + 1)
        got_len = [min(x, budget) for x in lens]
        assert c.dlen.tolist() == got_len
        dpos, dsc = c.dpos.cpu(), c.dscores.cpu()
        for b in range(2):
            for j in range(2):
                m = got_len[b]
                where = {int(x): s for s, x in enumerate(c.pos[b, j, :lens[b]])}
                kept = np.array([where[int(x)] for x in dpos[b, j, :m]])
                assert len(set(kept)) == m
                gone = np.setdiff1d(np.arange(lens[b]), kept)
                full = c.pos[b, j, :lens[b]].numpy()
                safe = (full < 4) | (full > full.max() - 30)
                assert not safe[gone].any()
                score = want[b, j].numpy()
                free = [s for s in kept if not safe[s]]
                if len(gone) and free:
                    assert score[gone].max() <= score[free].min() + 2 * margin
                idx = torch.from_numpy(kept)
                assert (dsc[b, j, :m].double() - want[b, j][idx]).abs().max() <= margin
                assert same(c.dk[b, j, :m], k[b, j][idx]) and same(c.dv[b, j, :m], v[b, j][idx])
        # on with the device's state
        c.k, c.v, c.scores, c.pos = c.dk.cpu(), c.dv.cpu(), dsc, dpos
        c.lens = got_len
    assert c.cache.flags() == [0, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rollout(dtype):
    rollout(dtype, 8)


def test_rollout_on_another_stream():
    rollout("bf16", 4, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rollout_in_a_graph(dtype):
    rollout(dtype, 6, graph=True)


def test_two_caches_on_two_streams():
    # calls of different caches at the same time share nothing
    cs = [Case("bf16", 128, b=2, hkv=2, g=3, cap=4000, lens=(4000, 1700), t=9, seed=i) for i in range(2)]
    want = [c.cache.attend(c.dq, c.dkn, c.dvn) for c in cs]
    ss = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        got = [c.cache.attend(c.dq, c.dkn, c.dvn, stream=s) for c, s in zip(cs, ss)]
    torch.cuda.synchronize()
    for (o, z), (p, y) in zip(want, got):
        assert torch.equal(o, p) and torch.equal(z, y)


def test_outputs_made_by_the_call_are_zero_behind_counts():
    # out and lse made by the call: zeros behind counts
    c = Case("bf16", 64, b=2, hkv=1, g=2, cap=40, lens=(40, 9), t=5)
    out, lse = c.cache.attend(c.dq, c.dkn, c.dvn, counts=ints([5, 2]))
    assert (out[1, :, 2:] == 0).all() and (lse[1, :, 2:] == 0).all()
    assert out.shape == c.dq.shape and lse.shape == (2, 2, 5)


# ---- many entries, long strides, graphs side by side --------------------------

@pytest.mark.parametrize("dtype,b,hkv,g,t", [("bf16", 2, 1, 3, 1), ("bf16", 5, 2, 2, 9),
                                             ("bf16", 33, 1, 2, 1), ("bf16", 70, 1, 1, 3),
                                             ("bf16", 70, 1, 3, 45), ("f32", 7, 1, 2, 1),
                                             ("f32", 70, 1, 1, 2)])
def test_parts_of_many_entries(dtype, b, hkv, g, t):
    # parts of very uneven entries; more entries than a wave has lanes
    lens = [int(x) for x in np.random.default_rng(b).integers(0, 120, b)]
    lens[b // 2] = 2900
    lens[-1] = 1333
    lens[0] = 0
    run_attend(Case(dtype, 64, b=b, hkv=hkv, g=g, cap=2900, lens=lens, t=t, seed=b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [3, 40])
def test_accumulate_of_many_entries(dtype, t):
    b = 70
    lens = [int(x) for x in np.random.default_rng(t).integers(0, 90, b)]
    lens[67], lens[3] = 600, 0
    rows = np.random.default_rng(5).integers(0, t, (b, t))
    counts = [min(n, t) for n in lens]
    run_accumulate(Case(dtype, 64, b=b, hkv=1, g=1, cap=600, lens=lens, t=t), rows=rows, counts=counts)


def test_append_and_evict_of_many_entries():
    b = 70
    lens = [int(x) for x in np.random.default_rng(8).integers(0, 60, b)]
    c = Case("bf16", 64, b=b, hkv=2, g=1, cap=64, lens=lens, t=5)
    rows, tpos = np.tile(np.arange(5), (b, 1)), np.tile(1000 + np.arange(5), (b, 1))
    k, v, sc, pos, new, flags = append_ref(c, rows, [5] * b, tpos)
    c.cache.append(c.dkn, c.dvn, positions=ints(tpos))
    torch.cuda.synchronize()
    assert c.dlen.tolist() == new and c.cache.flags() == flags
    assert same(c.dk, k) and same(c.dv, v)
    assert torch.equal(c.dscores.cpu(), sc) and torch.equal(c.dpos.cpu(), pos)
    run_evict(Case("bf16", 64, b=b, hkv=2, g=1, cap=64, lens=lens, t=1), 20, 2, 5)
    run_evict(Case("bf16", 64, b=b, hkv=2, g=1, cap=64, lens=lens, t=1), 20, 2, 5, other=1)


def far_apart(x, stride):
    """x [B, H, N, d] on the device with rows `stride` elements apart."""
    b, h, n, d = x.shape
    assert b == h == 1
    room = torch.empty((n - 1) * stride + d, dtype=x.dtype, device="cuda")
    view = room.as_strided((1, 1, n, d), (room.numel(), room.numel(), stride, 1))
    view.copy_(x)
    return view


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_32_bits(dtype):
    # rows 2^24 elements apart: the cache's slots and the new tokens' lie far behind 2^32 bytes
    far = 1 << 24
    c = Case(dtype, 64, b=1, hkv=1, g=2, cap=150, lens=(140,), t=5, fill=0.5)
    c.dk, c.dv, c.dkn, c.dvn = (far_apart(x, far) for x in (c.k, c.v, c.kn, c.vn))
    c.cache = S().KVCache(c.dk, c.dv, c.dlen, scores=c.dscores, positions=c.dpos)
    assert 149 * far * c.dk.element_size() > 2 ** 32
    run_attend(c)
    run_accumulate(c)
    c.scores = c.dscores.cpu()
    rows, tpos = np.arange(5)[None], np.arange(500, 505)[None]
    k, v, sc, pos, lens, flags = append_ref(c, rows, [5], tpos)
    c.cache.append(c.dkn, c.dvn, positions=ints(tpos))
    torch.cuda.synchronize()
    assert c.dlen.tolist() == lens and flags == [0]
    assert same(c.dk, k) and same(c.dv, v)
    c.k, c.v, c.scores, c.pos, c.lens = k, v, sc, pos, lens
    run_evict(c, 90, 4, 20)


@pytest.mark.parametrize("t", [134, 250])
def test_frame_of_far_apart_rows(t):
    # many rows: the shared tiles of both attention and accumulation
    far = 1 << 24
    c = Case("bf16", 64, b=1, hkv=1, g=1, cap=140, lens=(140,), t=t, fill=0.5)
    c.dk, c.dv = far_apart(c.k, far), far_apart(c.v, far)
    c.cache = S().KVCache(c.dk, c.dv, c.dlen, scores=c.dscores, positions=c.dpos)
    run_attend(c)
    run_accumulate(c)


def test_counts_are_clamped():
    c = Case("bf16", 64, b=3, hkv=1, g=2, cap=40, lens=(40, 9, 20), t=5)
    out, lse = c.cache.attend(c.dq, c.dkn, c.dvn)
    o2, z2 = torch.full_like(out, 7.0), torch.full_like(lse, -5.0)
    c.cache.attend(c.dq, c.dkn, c.dvn, counts=ints([99, 5, -4]), out=o2, lse=z2)
    assert torch.equal(out[:2], o2[:2]) and torch.equal(lse[:2], z2[:2])
    assert (o2[2] == 7.0).all() and (z2[2] == -5.0).all()


def test_one_cache_on_two_streams_and_two_graphs():
    # calls on one cache at the same time, each with a workspace of its own; graphs
    # of two caches replayed in turn
    cs = [Case("bf16", 128, b=2, hkv=2, g=3, cap=3000, lens=(3000, 700), t=9, seed=i) for i in range(2)]
    want = [c.cache.attend(c.dq, c.dkn, c.dvn) for c in cs]
    ss = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = [cs[0].cache.attend(c.dq, cs[0].dkn, cs[0].dvn, stream=s)
           for _ in range(5) for c, s in zip((cs[0], cs[0]), ss)]
    torch.cuda.synchronize()
    for o, z in got:
        assert torch.equal(o, want[0][0]) and torch.equal(z, want[0][1])
    graphs, outs = [], []
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.cache.attend(c.dq, c.dkn, c.dvn))
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        outs[i][0].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
