"""Plans of the gated feed-forward at the widths of the largest configuration, 8192 <-> 28,672 (csrc/glu_plan.h, asked on the CPU)."""
import pytest

pytest.importorskip("torch")
from tests.test_glu_plans import LARGE, MEDIUM, plans  # noqa: E402,F401


@pytest.mark.parametrize("n,F", [(8192, 28672), (28672, 8192)])
def test_plans_of_the_largest_widths(plans, n, F):  # noqa: F811
    for T in (1, 16, 33, 300, 1000, 2100, 4096, 8192):
        for bf16 in (True, False):
            p = plans(T, n, F, bf16)
            for name, parts in p.items():
                for q in parts:
                    rows = 16 if q["rows"] <= 16 else 32
                    groups = -(-F // 16) * -(-q["rows"] // rows) if q["ks"] else q["tiles"]
                    assert groups * max(q["ks"] * 64, 256) < 2 ** 32 or q["tile"] == LARGE, (T, name, q)
                    # partial sums are for results of few rows, and never larger than a weight in fp32
                    assert q["splits"] == 1 or q["splits"] * q["rows"] * n <= F * n, (T, name, q)
            # long calls: large tiles in every product, none split
            if bf16 and T >= 4096:
                assert all(q["tile"] <= MEDIUM and q["splits"] == 1 for parts in p.values() for q in parts)
                assert all(parts[0]["tile"] == LARGE for parts in p.values())
