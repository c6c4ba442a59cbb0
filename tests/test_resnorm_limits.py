"""Calls of the join that are refused on the host: gradients that share memory."""
import ctypes
import itertools

import pytest

pytest.importorskip("torch")
from paper_2608_26430_amd import binding  # noqa: E402
from tests.test_resnorm_pins import _packed  # noqa: E402

NAMES = ("dgate", "dpw", "dpb", "dw", "db")


def _bwd(T, n, groups, outs):
    """Status of a backward whose five vectors' gradients lie at `outs`.  (The pointers are never read: what is not refused here has
    no rows and is refused for its workspace, or none and no outputs.)"""
    q = 1 << 24
    d = dict(T=T, n=n, act=0, post=2, norm=2, gate=q, groups=groups, ldgate=n, res_scale=1.0, block_scale=1.0, post_eps=1e-5, eps=1e-5)
    p = ctypes.c_void_p(q)
    lib = binding._load()
    st = lib.ff_resnorm_bwd(_packed(**d), p, n, p, n, p, n, p, n, p, None, n, None, n, 0,
                            *(ctypes.c_void_p(outs.get(k)) for k in NAMES), None, 0, None)
    return binding._STATUS[st], lib.ff_last_error().decode()


@pytest.mark.parametrize("a,b", itertools.combinations(NAMES, 2))
@pytest.mark.parametrize("T", [0, 12])
def test_two_gradients_in_one_memory_are_refused(a, b, T):
    """One tensor for two vectors that a model shares: two workgroups would write, or add to, the same elements."""
    n, groups, at = 64, 3, 1 << 20
    for first, second in ((a, b), (b, a)):
        size = 4 * n * (groups if first == "dgate" else 1)
        for off in (0, 4, size - 4):
            st, text = _bwd(T, n, groups, {first: at, second: at + off})
            assert st == "FF_EINVAL" and "share" in text, (first, second, off, text)
    # side by side they are taken: the next check is that of the workspace
    if T:
        sizes = [4 * n * (groups if k == "dgate" else 1) for k in (a, b)]
        st, text = _bwd(T, n, groups, {a: at, b: at + sizes[0]})
        assert st == "FF_EINVAL" and "workspace" in text, text
