"""Every kernel that the linear layer's products choose among, by sizes whose plan names it: ragged tokens, outputs and sums, row
pitches, the whole epilogue, rows that are not finite.  Tolerances as in test_gpu_linear.py: small integers are exact."""
import pytest
import torch

import policy_reference as ref
from paper_2512_23353_amd import isopo

pytestmark = pytest.mark.gpu

CODE = {"f32": isopo.F32, "bf16": isopo.BF16}
# dtype, (tile, waves that split a tile's sum, whether workgroups do), (tokens, terms, outputs): the same for Y and for dX
KERNELS = (("bf16", (256, 1, False), (2803, 8, 8008)), ("bf16", (256, 1, False), (2803, 72, 8008)), ("bf16", (256, 1, False), (3001, 136, 4104)),
           ("bf16", (256, 1, False), (5000, 200, 4104)), ("bf16", (128, 1, False), (1100, 264, 520)), ("bf16", (128, 1, True), (70, 2056, 264)),
           ("f32", (128, 1, False), (2803, 8, 8012)), ("f32", (128, 1, False), (2803, 20, 8012)), ("f32", (128, 1, False), (4100, 72, 4108)),
           ("f32", (128, 1, False), (3001, 136, 4104)), ("f32", (128, 1, True), (200, 520, 4104)), ("f32", (64, 1, False), (700, 40, 520)),
           ("f32", (64, 1, True), (9, 520, 72)), ("f32", (64, 4, False), (70, 264, 264)), ("f32", (64, 4, True), (9, 2056, 72)),
           ("f32", (64, 8, False), (70, 1032, 4104)), ("f32", (64, 8, True), (9, 8200, 72)))


def _planned(dtype, kernel, n, d_in, d_out, backward):
    (p,) = isopo.linear_plan(n, d_in, d_out, CODE[dtype], backward)
    assert (p["tile"], p["sum_waves"], p["parts"] > 1) == kernel


def _integers(gen, shape, most, dtype, density=1.0):
    x = torch.randint(-most, most + 1, shape, generator=gen, device=gen.device, dtype=torch.int32)
    return (x * (torch.rand(shape, generator=gen, device=gen.device) < density)).to(ref.DTYPES[dtype])


def _pitched(x, extra):
    """The same values in rows that lie `extra` elements further apart, from the eighth element of a row on."""
    wide = torch.full((x.shape[0], x.shape[1] + extra), 3.0, dtype=x.dtype, device=x.device)
    wide[:, 8:8 + x.shape[1]] = x
    return wide, wide[:, 8:8 + x.shape[1]]


@pytest.mark.parametrize("dtype,kernel,size", KERNELS)
def test_forward(gpu_device, dtype, kernel, size):
    n, k, n_out = size
    _planned(dtype, kernel, n, k, n_out, False)
    gen = torch.Generator(device=gpu_device).manual_seed(n + k)
    X, W = _integers(gen, (n, k), 2, dtype), _integers(gen, (n_out, k), 2, dtype, min(1.0, 24 / k))
    b, R = _integers(gen, (n_out,), 9, dtype), _integers(gen, (n, n_out), 20, dtype)
    Wt = W.double().t().contiguous()
    z = X.double() @ Wt + b.double()
    assert z.abs().max() <= 250
    assert torch.equal(isopo.linear(X, W).double(), z - b.double())
    y = torch.clamp_min(z, 0) + R.double()
    Y, Z = isopo.linear(X, W, b, "relu", R, keep_z=True)
    assert torch.equal(Z.double(), z) and torch.equal(Y, y.to(Y.dtype))
    _, xp = _pitched(X, 24)
    store, rp = _pitched(R, 40)
    Y = isopo.linear(xp, W, b, "relu", residual=rp, Y=rp)
    assert Y is rp and torch.equal(rp, y.to(R.dtype))
    assert bool((store[:, :8] == 3.0).all()) and bool((store[:, 8 + n_out:] == 3.0).all())
    # a NaN or infinity among the last tokens, and one in a middle one, reach their rows alone
    W[:, k // 2] = 1.0
    Wt = W.double().t().contiguous()
    X[n // 2, k // 2], X[n - 1, k // 2] = float("nan"), float("inf")
    got, want = isopo.linear(X, W), X.double() @ Wt
    bad = torch.zeros(n, dtype=torch.bool, device=gpu_device)
    bad[n // 2] = bad[n - 1] = True
    assert torch.equal(got[~bad].double(), want[~bad])
    assert bool(torch.isnan(got[n // 2]).all()) and not torch.isfinite(got[n - 1]).any()


@pytest.mark.parametrize("dtype,kernel,size", KERNELS)
def test_backward(gpu_device, dtype, kernel, size):
    n, d_out, d_in = size
    _planned(dtype, kernel, n, d_in, d_out, True)
    gen = torch.Generator(device=gpu_device).manual_seed(n + d_out)
    dY, Z = _integers(gen, (n, d_out), 2, dtype), _integers(gen, (n, d_out), 3, dtype)
    W = _integers(gen, (d_out, d_in), 2, dtype, min(1.0, 24 / d_out))
    d = dY.double() * (Z > 0)
    dx = d @ W.double()
    assert dx.abs().max() <= 250
    for given in (dY, _pitched(dY, 24)[1]):
        Delta, dX, db = isopo.linear_backward(given, W, Z, "relu", need_db=True)
        assert torch.equal(Delta.double(), d) and torch.equal(dX.double(), dx) and torch.equal(db.double(), d.sum(0))
        _, dX, db = isopo.linear_backward(given, W, need_db=True)
        assert torch.equal(dX.double(), dY.double() @ W.double()) and torch.equal(db.double(), dY.double().sum(0))
    W[d_out // 2] = 1.0
    dY[n // 2, d_out // 2], dY[n - 1, d_out // 2] = float("nan"), float("inf")
    _, dX, _ = isopo.linear_backward(dY, W)
    bad = torch.zeros(n, dtype=torch.bool, device=gpu_device)
    bad[n // 2] = bad[n - 1] = True
    assert torch.equal(dX[~bad].double(), (dY.double() @ W.double())[~bad])
    assert bool(torch.isnan(dX[n // 2]).all()) and not torch.isfinite(dX[n - 1]).any()


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype,kernel,size", [c for c in KERNELS if c[2][1] in (136, 264, 520)])
def test_against_64_bits(gpu_device, dtype, kernel, size, act):
    n, k, n_out = size
    _planned(dtype, kernel, n, k, n_out, False)
    t, u = ref.DTYPES[dtype], ref.UNIT[dtype]
    gen = torch.Generator(device=gpu_device).manual_seed(n + k)
    mk = lambda *s: torch.randn(s, generator=gen, device=gpu_device)  # noqa: E731
    X, W, b, R = mk(n, k).to(t), (mk(n_out, k) * 2 * k ** -0.5).to(t), mk(n_out).to(t), mk(n, n_out).to(t)
    Y, Z = isopo.linear(X, W, b, act, R, keep_z=True)
    some = torch.cat([torch.arange(min(n, 150)), torch.arange(max(0, n - 150), n)]).to(gpu_device)
    y, z, s = ref.linear(X[some], W, b, act, R[some])
    sums = (k + 6) * 2.0 ** -24 * s
    assert bool(((Z[some].double().cpu() - z).abs() <= sums + u * (z.abs() + sums)).all())
    before = 1.13 * sums + 2.0 ** -20 * (z.abs() + sums) + 2.0 ** -24 * (y.abs() + 1)
    assert bool(((Y[some].double().cpu() - y).abs() <= before + u * (y.abs() + before)).all())
