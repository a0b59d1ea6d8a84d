"""Linear layers of more tokens than one launch takes."""
import pytest
import torch

from paper_2512_23353_amd import isopo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backward", (False, True))
def test_a_product_of_two_launches(gpu_device, backward):
    """The second launch has few tokens, which a call of their own would split into parts.  Small integers: results are exact.  34 GB of outputs."""
    k, n_out, more = 1024, 14336, 24
    d_in, d_out = (n_out, k) if backward else (k, n_out)
    most = isopo.linear_plan((1 << 31) - 1, d_in, d_out, isopo.BF16, backward)[0]["tokens"]
    n = most + more
    assert [p["tokens"] for p in isopo.linear_plan(n, d_in, d_out, isopo.BF16, backward)] == [most, more]
    assert isopo.linear_plan(more, d_in, d_out, isopo.BF16, backward)[0]["parts"] > 1
    gen = torch.Generator(device=gpu_device).manual_seed(3)
    X = torch.randint(-1, 2, (n, k), generator=gen, device=gpu_device, dtype=torch.int8).bfloat16()
    W = torch.randint(-2, 3, (d_out, d_in), generator=gen, device=gpu_device, dtype=torch.int8).bfloat16()
    W *= torch.rand(W.shape, generator=gen, device=gpu_device) < 24 / k
    if backward:
        _, Y, db = isopo.linear_backward(X, W, need_db=True)
        assert torch.equal(db.double(), sum((x.double().sum(0) for x in X.split(1 << 17)), torch.zeros(k, dtype=torch.float64, device=gpu_device)))
    else:
        Y = isopo.linear(X, W)
    torch.cuda.synchronize()
    Wt = (W if backward else W.t()).double().contiguous()
    for rows in (slice(0, 300), slice(most // 2, most // 2 + 300), slice(most - 300, n)):
        want = X[rows].double() @ Wt
        assert want.abs().max() <= 250 and torch.equal(Y[rows].double(), want), rows
