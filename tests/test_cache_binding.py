"""Host-side checks of the operators on a K/V cache beyond test_cache_abi.py: the
limits of their launches, their workspaces, gradients."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import test_cache_abi as A  # noqa: E402
from test_cache_abi import P, S, _ref, cache, tokens  # noqa: E402


def test_calls_that_would_be_refused_gradients():
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
    with pytest.raises(ValueError, match="grad"):
        c.attend(q, kn, kn)
