"""The launches that a linear layer's product is cut into, and the workspace that they share.  Host arithmetic: no GPU needed."""
import ctypes

import pytest

from paper_2512_23353_amd import isopo

# (d_in, d_out): widths whose last launch alone, of few tokens, would be split into parts
LAYERS = ((4096, 14336), (14336, 4096), (4096, 4096), (2048, 2048), (1536, 8960), (8960, 1536), (512, 50264), (16384, 64), (64, 16384), (8, 8))


def _whole(n, d_in, d_out, dtype, backward):
    """Tokens of a full launch of a product that is cut."""
    return isopo.linear_plan(n, d_in, d_out, dtype, backward)[0]["tokens"]


@pytest.mark.parametrize("dtype", (isopo.BF16, isopo.F32))
@pytest.mark.parametrize("backward", (False, True))
@pytest.mark.parametrize("d_in,d_out", LAYERS)
def test_a_cut_product_stays_in_its_workspace(d_in, d_out, dtype, backward):
    lib = isopo.load()
    workspace = lib.isopo_linear_backward_workspace if backward else lib.isopo_linear_workspace
    most = _whole((1 << 31) - 1, d_in, d_out, dtype, backward)
    assert most % 256 == 0
    for launches in (1, 2):
        for more in (1, 8, 24, 64, 128, 129, 512, 1000, 1024, 5000):
            n = launches * most + more
            if n >= 1 << 31:
                continue
            plan = isopo.linear_plan(n, d_in, d_out, dtype, backward)
            assert [p["tokens"] for p in plan] == [most] * launches + [more]
            assert max(p["workspace_end"] for p in plan) <= workspace(n, d_in, d_out, dtype)
            assert all(p["parts"] == 1 and p["workspace_end"] == 0 for p in plan)
    (alone,) = isopo.linear_plan(most, d_in, d_out, dtype, backward)
    assert alone["tokens"] == most and alone["workspace_end"] <= workspace(most, d_in, d_out, dtype)


@pytest.mark.parametrize("dtype", (isopo.BF16, isopo.F32))
@pytest.mark.parametrize("backward", (False, True))
def test_the_workspace_is_what_one_launch_needs(dtype, backward):
    lib, split = isopo.load(), 0
    for d_in, d_out in LAYERS:
        for n in (1, 2, 24, 64, 100, 128, 1000, 1024, 4096, 9999, 16384):
            (p,) = isopo.linear_plan(n, d_in, d_out, dtype, backward)
            rows, cols = n, d_in if backward else d_out
            assert p["tokens"] == n and p["tile"] in (64, 128, 256) and p["sum_waves"] in (1, 4, 8)
            have = (lib.isopo_linear_backward_workspace if backward else lib.isopo_linear_workspace)(n, d_in, d_out, dtype)
            if p["parts"] == 1:
                assert p["workspace_end"] == 0
                if not backward:
                    assert have == 0
                continue
            split += 1
            assert p["workspace_end"] == have
            assert have >= p["parts"] * rows * cols * 4
            if not backward:
                assert have == p["parts"] * rows * cols * 4
    assert split > 10


def test_plan_refuses():
    lib, info = isopo.load(), isopo.LinearPlanInfo()
    ok = (1 << 22, 4096, 14336, isopo.BF16, 0, 0, ctypes.byref(info))
    assert lib.isopo_linear_plan(*ok) == 0
    for i, bad, status in ((0, -1, 1), (0, 0, 1), (0, 1 << 31, 3), (1, 12, 3), (1, 0, 1), (2, 4, 3), (3, 5, 3), (5, -1, 1), (5, 256, 1), (5, 1 << 22, 1), (6, None, 1)):
        assert lib.isopo_linear_plan(*ok[:i], bad, *ok[i + 1:]) == status, (i, bad)
    assert isopo.linear_plan(0, 64, 64, isopo.BF16) == []


@pytest.mark.parametrize("n,d_out", ((1 << 30, 1 << 20), ((1 << 31) - 1, 1 << 21), (1 << 29, 1 << 21), ((1 << 31) - 1, (1 << 22) - 8), ((1 << 31) - 1, 8),
                                     (1 << 28, 4096)))
def test_the_workspace_of_the_largest_layers(n, d_out):
    """Rows per chunk of db's sums, 1024 workgroups of 256 columns over all of them, may pass 2^31."""
    rows = -(-n * -(-d_out // 256) // 1024)
    chunks = -(-n // (-(-rows // 8) * 8))
    need = isopo.load().isopo_linear_backward_workspace(n, 8, d_out, isopo.BF16)
    assert need == (chunks * d_out * 4 if chunks > 1 else 0)
