"""Host-side checks of the operators on a K/V cache beyond test_cache_abi.py: the
limits of their launches, workspaces, gradients."""
import ctypes

import pytest

import test_cache_abi as A
from test_cache_abi import S, _ref, cache, tokens


def size(fn, *args):
    n = ctypes.c_size_t(0)
    st = getattr(S.lib(), fn)(*args, ctypes.byref(n))
    return st, n.value, S.lib().sparsepr_last_error().decode()


def wide(heads, cap, dtype=S.F32):
    return cache(batch=1, heads_kv=heads, capacity=cap, dtype=dtype, stride_n=64, stride_h=64 * cap,
                 stride_b=64 * cap * heads)


def many(heads, n):
    return tokens(heads=heads, n=n, stride_n=0, stride_h=0, stride_b=0, kv_stride_n=0, kv_stride_h=0,
                  kv_stride_b=0, out_stride_n=64, out_stride_h=64 * n, out_stride_b=64 * n * heads)


@pytest.mark.parametrize("dtype,tile", [(S.F32, 32), (S.BF16, 128)])
def test_attention_of_more_rows_than_a_launch_holds_is_refused(dtype, tile):
    # 2^32 threads are 2^24 blocks of 256
    for heads, n, ok in ((7, 1 << 21, True), (7, 1 << 28, tile == 128), (4, 1 << 27, tile == 128)):
        assert heads * n < 1 << 31
        st, _, msg = size("sparsepr_cache_attend_workspace_size", _ref(wide(heads, 100, dtype)),
                          _ref(many(heads, n)))
        assert st == (0 if ok else 2), msg
        if not ok:
            assert "launch" in msg
            st, msg = A.attend(wide(heads, 100, dtype), many(heads, n))
            assert st == 2 and "launch" in msg


@pytest.mark.parametrize("dtype", [S.F32, S.BF16])
def test_weights_of_more_rows_than_a_launch_holds_are_refused(dtype):
    for heads, n, ok in ((7, 1 << 21, True), (3, 1 << 27, True), (4, 1 << 27, False), (7, 1 << 28, False)):
        c, t = wide(heads, 100, dtype), many(heads, n)
        st, _, msg = size("sparsepr_cache_accumulate_workspace_size", _ref(c), _ref(t), ctypes.c_int32(n))
        assert st == (0 if ok else 2), msg
        if not ok:
            assert "launch" in msg
            st, msg = A.accumulate(c, t, n_rows=n)
            assert st == 2 and "launch" in msg


def test_row_parts_of_an_accumulation_fit_a_launch():
    # 2^28 slots of a head are 2^20 blocks of 256 and 2^21 of 128: as many parts of the
    # rows as there is room for (a sum for each slot and part), down to one
    for dtype, heads, most in ((S.BF16, 1, 8), (S.BF16, 4, 3), (S.BF16, 9, 1), (S.F32, 4, 1)):
        st, n, msg = size("sparsepr_cache_accumulate_workspace_size", _ref(wide(heads, 1 << 28, dtype)),
                          _ref(many(heads, 3000)), ctypes.c_int32(3000))
        assert st == 0, msg
        sums = heads * (1 << 28) * 4
        assert n // sums == (most if most > 1 else 0)
    for dtype, heads in ((S.BF16, 16), (S.F32, 8)):
        st, _, msg = size("sparsepr_cache_accumulate_workspace_size", _ref(wide(heads, 1 << 28, dtype)),
                          _ref(many(heads, 3000)), ctypes.c_int32(3000))
        assert st == 2 and "launch" in msg


def test_eviction_of_more_slots_than_a_launch_holds_is_refused():
    # blocks of 4,096 slots and 1,024 threads: 2^22 of them
    for heads, ok in ((63, True), (64, False)):
        c = wide(heads, 1 << 28)
        st, _, msg = size("sparsepr_cache_evict_workspace_size", _ref(c), ctypes.c_int32(50))
        assert st == (0 if ok else 2), msg
    st, msg = A.evict(c, nbytes=1 << 62)
    assert st == 2 and "launch" in msg


def test_workspaces_of_split_calls_checked():
    # 4,000 slots are cut into parts, 80 rows are gathered: both need a workspace
    big = dict(capacity=4000, stride_h=4000 * 64, stride_b=4 * 4000 * 64)
    c, t = cache(**big), tokens(n=40, stride_h=40 * 64, stride_b=8 * 40 * 64, out_stride_h=40 * 64,
                                out_stride_b=8 * 40 * 64, kv_stride_h=40 * 64, kv_stride_b=4 * 40 * 64)
    st, need, _ = size("sparsepr_cache_attend_workspace_size", _ref(c), _ref(t))
    assert st == 0 and need > 0
    bare = cache(k=None, v=None, lengths=None, **big)
    assert size("sparsepr_cache_attend_workspace_size", _ref(bare), _ref(t))[:2] == (0, need)
    st, n_weigh, _ = size("sparsepr_cache_accumulate_workspace_size", _ref(c), _ref(t), ctypes.c_int32(40))
    assert st == 0 and n_weigh > 0
    for f, n, kw in ((A.attend, need, {}), (A.accumulate, n_weigh, dict(n_rows=40))):
        st, msg = f(c, t, nbytes=n - 1, **kw)
        assert st == 3 and "needs" in msg
        st, msg = f(c, t, ws=None, **kw)
        assert st == 1 and "workspace" in msg
        st, msg = f(c, t, ws=A.P + 8, **kw)
        assert st == 1 and "aligned" in msg


# --- the binding ------------------------------------------------------------

torch = pytest.importorskip("torch")


def test_tensors_that_require_gradients_are_refused():
    # the operators have no backward: an output without a graph would lose gradients
    q, kn = torch.zeros(2, 8, 5, 64), torch.zeros(2, 4, 5, 64)
    pos = torch.zeros(2, 5, dtype=torch.int32)
    lse = torch.zeros(2, 8, 5)
    leaf = {True: lambda x: x.clone().requires_grad_(), False: lambda x: x}
    for i in range(3):
        x = [leaf[i == j](y) for j, y in enumerate((q, kn, kn))]
        with pytest.raises(ValueError, match="grad"):
            A.host_cache().attend(*x)
    with pytest.raises(ValueError, match="grad"):
        A.host_cache().append(leaf[True](kn), kn, positions=pos)
    with pytest.raises(ValueError, match="grad"):
        A.host_cache().accumulate(leaf[True](q), lse)
    with pytest.raises(ValueError, match="grad"):
        A.host_cache(k=torch.zeros(2, 4, 100, 64).requires_grad_())
    with torch.no_grad():
        c = A.host_cache(k=torch.zeros(2, 4, 100, 64).requires_grad_())
        c._q(leaf[True](q))  # accepted
    for f in (lambda: c.attend(q, kn, kn), lambda: c.append(kn, kn, positions=pos),
              lambda: c.accumulate(q, lse), lambda: c.evict(5)):
        with pytest.raises(ValueError, match="k: requires grad"):
            f()


def test_sizes_beyond_32_bits_are_refused():
    # views of one row: their lengths would lose their upper bits on the way to the library
    far = 2 ** 32 + 1
    row = torch.zeros(2, 4, 1, 64)
    lengths = torch.zeros(2, dtype=torch.int32)
    c = A.HostCache(torch.zeros(2, 4, 100, 64), torch.zeros(2, 4, 100, 64), lengths)
    with pytest.raises(ValueError, match="k: shape"):
        A.HostCache(row.expand(2, 4, far, 64), row.expand(2, 4, far, 64), lengths)
    with pytest.raises(ValueError, match="k_new: shape"):
        c.append(row.expand(2, 4, far, 64), row.expand(2, 4, far, 64))
    with pytest.raises(ValueError, match="q: shape"):
        c.attend(row.expand(2, 4, far, 64), row.expand(2, 4, far, 64), row.expand(2, 4, far, 64))
    with pytest.raises(ValueError, match="q: shape"):
        c.attend(row[:, :1].expand(2, 4 * far, 1, 64), row, row)
