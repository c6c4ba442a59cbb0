"""Largest calls of dropout: checked on the host, before anything is launched."""
import ctypes

import pytest

pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402
from paper_2608_26430_amd import binding  # noqa: E402


@pytest.mark.parametrize("T,n", [(1 << 40, 1 << 28), (1 << 38, 1 << 28), (1 << 40, 129), ((1 << 19) + 1, 1 << 28)])
def test_more_blocks_than_their_numbers_have_bits_for_are_refused(T, n):
    """T ceil(n / 8) blocks are numbered in 64 bits, row starts too: sizes beyond every card are an error and no product that
    wraps.  (The pointer is never read: the call ends on the host.)"""
    p = ctypes.c_void_p(1 << 20)
    with pytest.raises(ff.FrameFTError) as ei:
        binding._check(binding._load().ff_dropout(T, n, binding.FF_F32, p, n, 0.5, 1, 0, None, None, n, p, n, None))
    assert ei.value.name == "FF_EINVAL" and "too many" in str(ei.value)
