"""The gated feed-forward at the widths of the largest configuration, 8192 <-> 28,672, from one token to some thousand: forward, kept and
made again, all gradients, against the definitions in 64 bits (references and bounds of test_gpu_glu.py)."""
import pytest

torch = pytest.importorskip("torch")
from tests.test_gpu_glu import data, whole  # noqa: E402

pytestmark = pytest.mark.gpu
SIZES = [(1, 8192, 28672), (16, 8192, 28672), (300, 8192, 28672), (2100, 8192, 28672), (130, 28672, 8192)]


@pytest.mark.parametrize("T,n,F", SIZES)
def test_largest_widths(T, n, F):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    if torch.cuda.mem_get_info()[0] < 60 * 2 ** 30:
        pytest.skip("needs 60 GiB")
    whole(data(T, n, F, "bf16", dev, T, adapters=T != 16), "silu" if T != 300 else "gelu_tanh")
