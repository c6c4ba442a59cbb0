"""Largest vocabularies of the head's loss: checked on the host, before a device is needed."""
import pytest

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("want", [dict(want_dh=True), dict(want_dw=True), dict(want_dh=True, want_dw=True)])
def test_gradients_of_vocabularies_past_a_tiles_range_are_refused(dtype, want):
    """dH's tiles have 256 rows of P (128 in fp32), a row as long as the vocabulary: with 2^22 entries the place of a tile's
    last piece fits 31 bits, with more it would not, and loads would read other places of P."""
    assert ff.xent_workspace(1, 64, 1 << 22, dtype, device="cpu", **want).nbytes > 0
    for V in ((1 << 22) + 1, 1 << 24):
        with pytest.raises(ff.FrameFTError) as ei:
            ff.xent_workspace(1, 64, V, dtype, device="cpu", **want)
        assert ei.value.name == "FF_EINVAL" and "V=" in str(ei.value)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_loss_alone_takes_larger_ones(dtype):
    assert ff.xent_workspace(1, 64, 1 << 24, dtype, device="cpu").nbytes > 0
    with pytest.raises(ff.FrameFTError):
        ff.xent_workspace(1, 64, (1 << 24) + 1, dtype, device="cpu")
