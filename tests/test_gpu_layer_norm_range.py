"""Layer norm of rows at the ends of what fp32 holds: rows that are no numbers, rows whose squares or sums are beyond it, and rows far from zero."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_layer_norm import types

pytestmark = pytest.mark.gpu

# a lane to a row's vector, part of a wavefront, a wavefront, workgroups of each size, rows beyond the registers
WIDTHS = [1, 3, 9, 47, 100, 300, 1000, 1501, 5000, 9001, 16_384, 32_768, 40_000]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_statistics_of_rows_that_are_no_numbers_are_none(d, dtype):
    import torch
    inf, nan = float("inf"), float("nan")
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(7, d, generator=gen, device="cuda").to(types()[dtype])
    x[0, d // 2], x[1, 0], x[2, d - 1], x[3, d // 3] = inf, -inf, nan, -nan
    x[4, :] = inf
    stats = torch.empty(7, 2, device="cuda")
    y = gp.layer_norm_tensors(x, stats=stats)
    assert bool(stats[:5, 1].isnan().all()) and not bool(stats[:5, 0].isfinite().any()) and bool(y[:5].isnan().all())
    assert bool(stats[5:].isfinite().all()) and bool(y[5:].isfinite().all())
    want = gp.layer_norm_tensors(x[5:].contiguous(), stats=torch.empty(2, 2, device="cuda"))
    assert torch.equal(y[5:], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [d for d in WIDTHS if d >= 100])
def test_rows_far_from_zero_lose_nothing(d, dtype):
    """u = 2^-24.  Rows in registers: the first mean is off by at most e = 52 u mean|x| (50 u of a sum, two roundings), and x less it is exact or off by u of itself; the mean of
    what is left is off by 52 u of its terms, f = 53 u (mean|x - m| + e).  The squares are of terms off by that mean, off by 54 u of themselves: of variance + e^2, taken from which
    the mean's square is off by 104 u e (mean|x - m| + e): so r, by half of it over variance + eps, and 3 u.  h = (x - m) r is off by r f, r's part and 2 u, y by |w| times
    that, two roundings of |h w|, one of y, and half a step of its type.  Rows beyond them have their mean in two parts, of which the second is off by u of itself, u^2 mean|x|,
    and x - m by 2 u of itself; the squares are off by 4 u and a rounding, added up in fp64, r by half of that and 4 u."""
    import torch
    from oracle import answers
    from test_gpu_layer_norm import U, half_step, wide
    gen = torch.Generator(device="cuda").manual_seed(d)
    spread = torch.tensor([[1e-2], [1.0], [0.3], [30.0]], device="cuda")
    far = torch.tensor([[1e4], [-3e5], [1e3], [-1e6]], device="cuda")
    x = (far + spread * torch.randn(4, d, generator=gen, device="cuda")).to(types()[dtype])
    w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
    stats = torch.empty(4, 2, device="cuda")
    for out_dtype in (torch.float32, torch.bfloat16):
        y = gp.layer_norm_tensors(x, w, b, eps=1e-6, out_dtype=out_dtype, stats=stats)
        X, W = wide(x), np.abs(wide(w))
        want, s = answers.layer_norm(X, wide(w), wide(b), float(np.float32(1e-6)))
        m, r = s[:, :1], s[:, 1:]
        h = np.abs((X - m) * r)
        if d <= (16_384 if dtype == "f32" else 32_768):
            near = np.abs(X - m).mean(1, keepdims=True)
            e = 52 * U * np.abs(X).mean(1, keepdims=True)
            f = 53 * U * (near + e)
            variance = ((X - m) ** 2).mean(1, keepdims=True)
            of_r = (54 * U * (variance + e ** 2) + 104 * U * e * (near + e)) * r ** 2 / 2 + 3 * U
        else:
            f, of_r = U ** 2 * np.abs(X).mean(1, keepdims=True), 7 * U
        off_h = r * f + h * of_r + (2 if d <= 16_384 else 3) * U * h
        bound = W * off_h + 2 * U * h * W + U * np.abs(want) + half_step(y) * np.abs(want)
        off = np.abs(wide(y) - want)
        assert (off <= bound).all(), f"worst {np.max(off / bound):.2f} of the bound"
        assert (np.abs(wide(stats)[:, :1] - m) <= U * np.abs(m) * 2 + f).all() and (np.abs(wide(stats)[:, 1:] - r) <= r * (of_r + U)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_whose_squares_or_sums_are_beyond_fp32(d, dtype):
    """u = 2^-24.  The sums are taken in fp64; x - m is rounded once, r off by 3 u (the variance, its root, the quotient), h = (x - m) r by 5 u with its own rounding, y by two
    roundings of |h w|, one of itself, and half a step of its type.  The statistics are rounded once, r below the least normal number by 2^-149 besides.  A row of one value is the bias."""
    import torch
    from oracle import answers
    from test_gpu_layer_norm import U, check_backward, half_step, wide
    gen = torch.Generator(device="cuda").manual_seed(d)
    ty = types()[dtype]
    most = torch.finfo(ty).max
    x = torch.randn(12, d, generator=gen, device="cuda").clamp(-3, 3)
    x[0] *= 1e25
    x[1] = x[1] * 1e30 + 1e32
    x[2] *= 1.1e38                                                      # squares and sums
    x[3] = torch.where(x[3] > 0, most, -most)                           # of both signs: x - m is beyond it too
    x[4] = most                                                         # one value
    x[5] = -most
    x[5, d // 2] = -most * (1 - 2.0 ** -7)                              # but for one, a step of bf16 off
    x[6] = 1e20 * torch.randint(0, 2, (d,), generator=gen, device="cuda")
    x[7] = 0.0
    x[7, d - 1] = most
    x[8] *= -1e21
    x[9] *= 1e22
    x = x.to(ty)
    w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
    for eps in (1e-5, 1e30):
        eps = float(np.float32(eps))
        alone = [gp.layer_norm_tensors(x[i:i + 1], w, b, eps=eps) for i in (10, 11)]
        for out_dtype in (torch.float32, torch.bfloat16):
            stats = torch.empty(12, 2, device="cuda")
            y = gp.layer_norm_tensors(x, w, b, eps=eps, out_dtype=out_dtype, stats=stats)
            X, W = wide(x), np.abs(wide(w))
            want, s = answers.layer_norm(X, wide(w), wide(b), eps)
            m, r = s[:, :1], s[:, 1:]
            h = np.abs((X - m) * r)
            bound = W * 6 * U * h + 2 * U * h * W + U * np.abs(want) + half_step(y) * np.abs(want) + 1e-37
            off = np.abs(wide(y) - want)
            assert (off <= bound)[:10].all(), f"worst {(off / bound)[:10].max(1)} of the bound"
            assert (np.abs(wide(stats) - s)[:10] <= 4 * U * np.abs(s[:10]) + 2.0 ** -149).all()
            assert torch.equal(y[4], b.to(out_dtype)) and bool(y.isfinite().all())
            if out_dtype == ty:  # the rows beside them are left alone
                assert torch.equal(y[10:], torch.cat(alone))
                again = x.clone()
                assert torch.equal(gp.layer_norm_tensors(again, w, b, eps=eps, out=again), y)
        g = torch.randn(12, d, generator=gen, device="cuda")
        fine = [0, 1, 6, 8, 9]
        dx, _, _ = gp.layer_norm_grad_tensors(g, x, stats, w)
        check_backward((dx[fine], None, None), g[fine], x[fine], stats[fine], w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_one_value_and_rows_a_step_from_it(d, dtype):
    """The bounds of rows far from zero, where a row in registers has its first mean off by no more than 6 sqrt(variance + eps) (it is done in fp64 from the square of that,
    32 times variance + eps, on): e is the lesser of the two.  In 80 bits, since fp64 leaves a step of 2^-53 of the mean, times r."""
    import torch
    from test_gpu_layer_norm import U, wide
    gen = torch.Generator(device="cuda").manual_seed(d)
    ty = types()[dtype]
    step = torch.finfo(ty).eps
    values = torch.tensor([1.1, -7.3e2, 1.37e4, -1.37e6, 1.37e8, 1.37e10, -1.37e12, 1.37e15, 1.37e18, 1.3e25, 3e38], device="cuda").to(ty).float()
    one = values[:, None].expand(-1, d)
    some = (torch.rand(len(values), d, generator=gen, device="cuda") < 0.3).float()
    last = (torch.arange(d, device="cuda") == d - 1).float().expand(len(values), d)
    x = torch.cat([one, one * (1 - step * some), one * (1 - 2 * step * last)]).to(ty)
    w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
    stats = torch.empty(len(x), 2, device="cuda")
    for eps in (1e-5, 1e-12):
        y = gp.layer_norm_tensors(x, w, b, eps=eps, out_dtype=torch.float32, stats=stats)
        X, W = wide(x).astype(np.longdouble), np.abs(wide(w))
        m = X.mean(1, keepdims=True)
        m = m + (X - m).mean(1, keepdims=True)
        v = ((X - m) ** 2).mean(1, keepdims=True) + np.longdouble(np.float32(eps))
        r = 1 / np.sqrt(v)
        want = ((X - m) * r).astype(np.float64) * wide(w) + wide(b)
        m, v, r, h = (a.astype(np.float64) for a in (m, v, r, np.abs((X - m) * r)))
        near = np.abs(X - m).mean(1, keepdims=True).astype(np.float64)
        e = np.minimum(52 * U * np.abs(m), 6 * np.sqrt(v))
        f = 53 * U * (near + e)
        of_r = (54 * U * (v + e ** 2) + 104 * U * e * (near + e)) * r ** 2 / 2 + 4 * U
        bound = W * (r * f + h * of_r + 3 * U * h) + 2 * U * h * W + 2 * U * np.abs(want) + U * np.abs(wide(b)) + 1e-37
        off = np.abs(wide(y) - want)
        assert (off <= bound).all(), f"worst {(off / bound).max(1)} of the bound"
        assert (np.abs(wide(stats)[:, 1:] - r) <= r * (of_r + U) + 2.0 ** -149).all() and (np.abs(wide(stats)[:, :1] - m) <= 2 * U * np.abs(m) + f).all()
