"""The training operators on the GPU against their definitions in 64 bits.

Tolerances.  A looked-up row is one fp32 product, rounded once: equal bits.  A gradient row of t terms is a sum in fp32 in some
order: at most t roundings of 2^-24 of the terms' magnitudes (and one for the scale), then one of the result (2^-24, or 2^-8 in bf16).
Newton-Schulz steps: with operands of 22 bits, step k leaves an error of a few 2^-22 of |X_k|, which the steps after it stretch by at
most the polynomial's largest slope L each: 4 * 2^-22 * sum_k L^(steps - k) |X_k| / |X_steps| in the Frobenius norm, and 2^-9 for a
result in bf16.  (Operands of 11 bits would be a thousand times that.)
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import training

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}


def padded(rows, cols, ld, dtype, skew=0, fill=float("nan")):
    """A (rows, cols) view with rows ld elements apart, `skew` elements into its memory; the rest is `fill`."""
    import torch
    flat = torch.full((rows * ld + skew + 64,), fill, dtype=dtype, device="cuda")
    return flat, flat[skew:skew + rows * ld].view(rows, ld)[:, :cols]


def same_bits(a, b):
    import torch
    assert a.dtype == b.dtype and a.shape == b.shape
    return torch.equal(a.contiguous().view(torch.int16 if a.element_size() == 2 else torch.int32),
                       b.contiguous().view(torch.int16 if a.element_size() == 2 else torch.int32))


# ---- lookup ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("kinds", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("N,V,d,pad,skew", [(1, 1, 1, 0, 0), (5, 3, 2, 1, 1), (1, 7, 128, 0, 0), (3, 9, 3, 0, 1), (77, 50, 4, 0, 0), (64, 11, 5, 0, 0),
                                            (130, 1000, 8, 3, 1), (257, 40, 47, 0, 1), (1000, 333, 100, 5, 3), (65, 13, 129, 0, 0),
                                            (33, 77, 602, 2, 0), (4096, 500, 256, 0, 0), (9, 5, 4097, 0, 1)])
def test_lookup(N, V, d, pad, skew, kinds, index):
    import torch
    ty = types()
    rng = np.random.default_rng(N * 31 + d)
    _, table = padded(V, d, d + pad, ty[kinds[0]], skew)
    table.copy_(torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32)))
    tokens = torch.from_numpy(rng.integers(-2, V + 2, N)).to(ty[index]).cuda()
    flat, out = padded(N, d, d + 2 * pad, ty[kinds[1]], skew, fill=7.0)
    for scale in (1.0, -0.37):
        got = gp.embedding_tensors(table, tokens, scale=scale, out=out)
        assert got is out
        known = (tokens >= 0) & (tokens < V)
        want = (table.float()[tokens.long().clamp(0, V - 1)] * torch.tensor(scale, device="cuda") * known[:, None].float())
        want = torch.where(known[:, None], want, torch.zeros_like(want)).to(ty[kinds[1]])
        assert same_bits(out, want)
        if pad:  # between the rows, before and behind them: untouched
            flat[skew:skew + N * (d + 2 * pad)].view(N, -1)[:, :d] = 7.0
            assert bool((flat == 7.0).all())


def test_lookup_against_the_oracle():
    import torch
    rng = np.random.default_rng(5)
    table, tokens = rng.normal(size=(40, 19)).astype(np.float32), rng.integers(-1, 41, 100)
    got = gp.embedding_tensors(torch.from_numpy(table).cuda(), torch.from_numpy(tokens).cuda(), scale=0.5).cpu().numpy()
    assert np.array_equal(got, training.embedding(table, tokens, 0.5))


def test_lookup_keeps_the_shape_of_tokens_and_takes_none():
    import torch
    table = torch.randn(10, 6, device="cuda")
    tokens = torch.randint(0, 10, (3, 4), device="cuda")
    assert torch.equal(gp.embedding_tensors(table, tokens), table[tokens])
    assert gp.embedding_tensors(table, tokens[:0].contiguous()).shape == (0, 4, 6)
    far = torch.tensor([2 ** 40, -2 ** 63, 2 ** 32 + 1, 3], device="cuda")  # (2^32 + 1 is no 1)
    assert torch.equal(gp.embedding_tensors(table, far), torch.cat([torch.zeros(3, 6, device="cuda"), table[3:4]]))


def test_special_values_of_the_table():
    import torch
    table = torch.tensor([[float("inf"), float("nan"), -0.0, 3e38]], device="cuda")
    got = gp.embedding_tensors(table, torch.tensor([0, -1], device="cuda"), scale=2.0)
    assert got[0, 0] == float("inf") and got[0, 1].isnan() and got[0, 3] == float("inf") and torch.equal(got[1], torch.zeros(4, device="cuda"))
    nothing = gp.embedding_tensors(table, torch.tensor([-1], device="cuda"), scale=float("inf"))
    assert torch.equal(nothing, torch.zeros(1, 4, device="cuda"))


def test_lookup_and_gradient_past_32_bit_offsets():
    import torch
    V, d = 17_000_003, 260   # 4.4e9 elements of bf16
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 16_500_000, V - 1, 9_000_001], device="cuda")
    table[rows] = torch.randn(4, d, device="cuda").bfloat16()
    assert torch.equal(gp.embedding_tensors(table, rows), table[rows])
    up = torch.randn(4, d, device="cuda").bfloat16()
    gp.embedding_grad_tensors(rows.to(torch.int32), up, V, out=table)
    assert torch.equal(table[rows], up)
    assert int(torch.count_nonzero(table[16_500_001:V - 1])) == 0 and int(torch.count_nonzero(table[1:9_000_001])) == 0


# ---- gradient ----------------------------------------------------------------------------------------------

def check_gradient(got, tokens, up, V, scale, before=None):
    want, size, terms = training.embedding_grad(tokens.cpu().numpy(), up.float().cpu().numpy(), V, scale)
    if before is not None:
        want, size = want + before, size + np.abs(before)
    last = 2.0 ** -24 if got.element_size() == 4 else 2.0 ** -8
    bound = (terms[:, None] + 2) * 2.0 ** -24 * size + last * np.abs(want) + 1e-37
    err = np.abs(got.float().cpu().numpy() - want)
    assert (err <= bound).all(), f"worst {np.nanmax(err / bound):.2f} of the bound"


def tokens_of(kind, N, V, rng):
    if kind == "uniform":
        return rng.integers(0, V, N)
    if kind == "one":      # every position names one row
        return np.full(N, V // 2)
    if kind == "none":
        return np.full(N, -1)
    if kind == "hot":      # half of them name one row, some name none
        t = rng.integers(0, V, N)
        t[rng.random(N) < 0.5] = V - 1
        t[rng.random(N) < 0.1] = V
        return t
    if kind == "sorted":
        return np.sort(rng.integers(0, V, N))
    return np.arange(N)[::-1] % V


@pytest.mark.parametrize("tokens_kind", ["uniform", "one", "none", "hot", "sorted", "falling"])
@pytest.mark.parametrize("N,V,d", [(1, 1, 1), (2, 3, 4), (15, 5, 47), (16, 16, 8), (17, 300, 128), (64, 2, 3), (1000, 70, 100), (1025, 5000, 33),
                                   (4096, 257, 64), (20_011, 47, 47), (70_001, 65_536, 16)])
def test_gradient(N, V, d, tokens_kind):
    import torch
    rng = np.random.default_rng(N + V)
    tokens = torch.from_numpy(tokens_of(tokens_kind, N, V, rng)).to(torch.int32).cuda()
    up = torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)).cuda()
    out = torch.full((V, d), float("nan"), device="cuda")
    gp.embedding_grad_tensors(tokens, up, V, scale=0.3, out=out)
    check_gradient(out, tokens, up, V, np.float32(0.3).astype(np.float64))


@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("kinds", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,V,d,pad,skew", [(600, 41, 1, 0, 1), (600, 41, 5, 1, 1), (3000, 900, 47, 0, 1), (2500, 30, 100, 4, 0), (900, 77, 130, 3, 1),
                                            (500, 29, 602, 1, 1), (300, 11, 1031, 0, 0)])
def test_gradient_types_and_strides(N, V, d, pad, skew, kinds, accumulate, index):
    import torch
    ty = types()
    rng = np.random.default_rng(d)
    tokens = torch.from_numpy(rng.integers(-1, V - 3, N)).to(ty[index]).cuda()   # (the last rows have no token)
    _, up = padded(N, d, d + pad, ty[kinds[0]], skew)
    up.copy_(torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)))
    flat, out = padded(V, d, d + 2 * pad, ty[kinds[1]], skew, fill=0.25)
    ws = torch.full((gp.gp_embedding_grad_workspace(N, V, d),), 255, dtype=torch.uint8, device="cuda")
    gp.embedding_grad_tensors(tokens, up, V, scale=2.0, out=out, accumulate=accumulate, workspace=ws)
    check_gradient(out, tokens, up, V, 2.0, before=0.25 if accumulate else None)
    first = out.clone()
    flat[skew:skew + V * (d + 2 * pad)].view(V, -1)[:, :d] = 0.25
    assert bool((flat == 0.25).all())                                            # nothing beside the rows was written
    gp.embedding_grad_tensors(tokens, up, V, scale=2.0, out=out, accumulate=accumulate)
    assert same_bits(out, first)


@pytest.mark.parametrize("N,V,d,tokens_kind", [(262_143, 1000, 16, "hot"), (262_145, 3, 20, "uniform"), (600_000, 2_000_000, 8, "uniform"),
                                               (1_000_003, 200_000, 12, "one")])
def test_gradient_of_long_lists(N, V, d, tokens_kind):
    import torch
    rng = np.random.default_rng(7)
    tokens = torch.from_numpy(tokens_of(tokens_kind, N, V, rng)).to(torch.int32).cuda()
    up = torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)).cuda()
    out = gp.embedding_grad_tensors(tokens, up, V)
    check_gradient(out, tokens, up, V, 1.0)
    assert same_bits(out, gp.embedding_grad_tensors(tokens, up, V))


def test_a_gradient_row_with_infinity_or_nan_stays_alone():
    import torch
    tokens = torch.tensor([3, 1, 3, 2, -1, 1], device="cuda")
    up = torch.ones(6, 9, device="cuda")
    up[0, 2], up[3, 4], up[4] = float("inf"), float("nan"), float("nan")
    got = gp.embedding_grad_tensors(tokens, up, 5)
    want = torch.tensor([0.0, 2.0, 1.0, 2.0, 0.0], device="cuda")[:, None].repeat(1, 9)
    want[3, 2], want[2, 4] = float("inf"), float("nan")
    assert torch.allclose(got, want, rtol=0, atol=0, equal_nan=True)


def test_no_tokens():
    import torch
    tokens, up = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 7, device="cuda")
    out = torch.ones(5, 7, device="cuda")
    gp.embedding_grad_tensors(tokens, up, 5, out=out, accumulate=True)
    assert bool((out == 1).all())
    gp.embedding_grad_tensors(tokens, up, 5, out=out)
    assert bool((out == 0).all())


def test_gradient_agrees_with_differences():
    """<lookup(table + D), up> - <lookup(table), up> = <grad, D>: the lookup is linear."""
    import torch
    rng = np.random.default_rng(3)
    table, step = (torch.from_numpy(rng.integers(-8, 9, (50, 21)).astype(np.float32)).cuda() for _ in range(2))   # (exact in fp32)
    tokens = torch.from_numpy(rng.integers(-1, 51, 400)).cuda()
    up = torch.from_numpy(rng.integers(-8, 9, (400, 21)).astype(np.float32)).cuda()
    moved = gp.embedding_tensors(table + step, tokens, scale=0.5) - gp.embedding_tensors(table, tokens, scale=0.5)
    grad = gp.embedding_grad_tensors(tokens, up, 50, scale=0.5)
    assert float((moved.double() * up.double()).sum()) == float((grad.double() * step.double()).sum())


# ---- Newton-Schulz -------------------------------------------------------------------------------------------

def tolerance(iterates, steps, coeff, out_bytes):
    coeff = np.broadcast_to(np.asarray(coeff, dtype=np.float64), (steps, 3))
    s = np.linspace(0.0, 1.25, 2001)
    slope = [np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max() for a, b, c in coeff]
    norms = [np.linalg.norm(x) for x in iterates]
    total = sum(np.prod(slope[k:]) * norms[k] for k in range(steps + 1)) / norms[-1]
    return 4 * 2.0 ** -22 * total + (2.0 ** -9 if out_bytes == 2 else 0.0)


def check_direction(got, G, steps=5, coeff=training.COEFF, eps=1e-7):
    iterates = training.newton_schulz(G.double().cpu().numpy(), steps, coeff, eps)
    err = np.linalg.norm(got.double().cpu().numpy() - iterates[-1]) / np.linalg.norm(iterates[-1])
    tol = tolerance(iterates, steps, coeff, got.element_size())
    assert err <= tol, f"{err:.3g} against {tol:.3g}"


def gradient_like(shape, rng, floor=0.2):
    """A few strong directions over a floor of noise."""
    k = max(1, min(shape) // 8)
    return 1e-3 * (rng.normal(size=(shape[0], k)) @ rng.normal(size=(k, shape[1])) + floor * rng.normal(size=shape))


SHAPES = [(1, 1), (1, 7), (7, 1), (16, 16), (16, 40), (63, 65), (64, 64), (65, 63), (128, 128), (130, 257), (256, 40), (40, 256), (256, 256), (602, 256),
          (100, 1023), (511, 513)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize(shape, dtype):
    import torch
    rng = np.random.default_rng(shape[0])
    for G in (rng.normal(size=shape), gradient_like(shape, rng)):
        G = torch.from_numpy(G).to(types()[dtype]).cuda()
        check_direction(gp.orthogonalize_tensors(G), G)


@pytest.mark.parametrize("shape", [(300, 1100), (1500, 700), (1024, 1024)])
def test_orthogonalize_larger(shape):
    import torch
    G = torch.from_numpy(gradient_like(shape, np.random.default_rng(4))).float().cuda()
    check_direction(gp.orthogonalize_tensors(G), G)


@pytest.mark.parametrize("steps,coeff", [(1, (1.5, -0.5, 0.0)), (2, (3.0, -16 / 5, 6 / 5)), (3, [(4.0, -6.0, 2.5), (3.0, -3.5, 1.4), (15 / 8, -10 / 8, 3 / 8)]),
                                         (8, (15 / 8, -10 / 8, 3 / 8)), (2, (0.0, 0.0, 0.0)), (4, (30.0, 0.0, 0.0)), (1, (-2.0, 1.0, 0.5))])
@pytest.mark.parametrize("shape", [(70, 90), (90, 70)])
def test_other_polynomials(shape, steps, coeff):
    import torch
    G = torch.from_numpy(gradient_like(shape, np.random.default_rng(6))).float().cuda()
    got = gp.orthogonalize_tensors(G, steps=steps, coeff=coeff)
    if not np.any(coeff):
        assert bool((got == 0).all())
    else:
        c32 = np.asarray(coeff, dtype=np.float32).astype(np.float64)
        check_direction(got, G, steps, c32)


@pytest.mark.parametrize("power", [-30, -12, 12, 30])
def test_any_magnitude(power):
    import torch
    G = torch.from_numpy(gradient_like((48, 130), np.random.default_rng(8)) * 10.0 ** power).float().cuda()
    check_direction(gp.orthogonalize_tensors(G, eps=0.0), G, eps=0.0)


def test_eps_rules_over_a_small_matrix_and_zero_stays_zero():
    import torch
    G = torch.from_numpy(np.random.default_rng(9).normal(size=(20, 30)) * 1e-9).float().cuda()
    check_direction(gp.orthogonalize_tensors(G, eps=1e-7), G, eps=1e-7)
    assert bool((gp.orthogonalize_tensors(torch.zeros(20, 30, device="cuda")) == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(33, 70), (70, 33), (200, 200)])
def test_batches_strides_and_in_place(shape, dtype):
    import torch
    rng = np.random.default_rng(10)
    ty = types()[dtype]
    G = torch.from_numpy(np.stack([gradient_like(shape, rng) for _ in range(3)])).to(ty).cuda()
    alone = torch.stack([gp.orthogonalize_tensors(g) for g in G])
    assert same_bits(gp.orthogonalize_tensors(G), alone)
    # matrices side by side in long rows, from an odd address; the rest is left alone
    flat = torch.full((1 + shape[0] * (3 * shape[1] + 5),), 9.0, dtype=ty, device="cuda")
    wide = flat[1:].view(shape[0], 3 * shape[1] + 5)
    side = wide[:, :3 * shape[1]].unflatten(1, (3, shape[1])).permute(1, 0, 2)
    side.copy_(G)
    ws = torch.full((gp.gp_orthogonalize_workspace(*shape, 3),), 255, dtype=torch.uint8, device="cuda")
    gp.orthogonalize_tensors(side, out=side, workspace=ws)
    assert same_bits(side, alone)
    assert bool((wide[:, 3 * shape[1]:] == 9.0).all()) and float(flat[0]) == 9.0
    one = G[0].clone()
    gp.orthogonalize_tensors(one, out=one)
    assert same_bits(one, alone[0])
    same = gp.orthogonalize_tensors(G[:1].expand(2, *shape))   # one matrix read twice
    assert same_bits(same, alone[:1].expand(2, *shape).contiguous())


def test_a_matrix_with_nan_or_infinity_spoils_no_other():
    import torch
    G = torch.from_numpy(np.random.default_rng(11).normal(size=(4, 50, 80))).float().cuda()
    want = gp.orthogonalize_tensors(G)
    G[1, 3, 4], G[2, 0, 0] = float("nan"), float("inf")
    got = gp.orthogonalize_tensors(G)
    assert bool(got[1].isnan().all()) and bool(got[2].isnan().all())
    assert same_bits(got[0], want[0]) and same_bits(got[3], want[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(1, 1), (256, 40), (96, 130), (130, 96)])
def test_muon_step(shape, nesterov, dtype):
    import torch
    rng = np.random.default_rng(12)
    W, M = (torch.from_numpy(x).float().cuda() for x in (rng.normal(size=shape) / shape[0] ** 0.5, 5 * gradient_like(shape, rng)))
    G = torch.from_numpy(gradient_like(shape, rng)).to(types()[dtype]).cuda()
    lr, mu, wd = (float(np.float32(x)) for x in (0.02, 0.95, 0.1))
    W2, M2 = gp.muon_step_tensors(W, M, G, lr, mu, wd, nesterov, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    w, m, g = (x.double().cpu().numpy() for x in (W, M, G))
    want_W, want_M = training.muon_step(w, m, g, lr, mu, wd, nesterov)
    # M: two roundings; W: the direction's tolerance (U itself has three roundings, which the steps stretch no further than
    # they do their own), times lr, and three roundings of its own
    assert (np.abs(M2.double().cpu().numpy() - want_M) <= 2.0 ** -23 * (np.abs(mu * m) + np.abs(g))).all()
    iterates = training.newton_schulz(g + mu * want_M if nesterov else want_M)
    tol = lr * 2 * tolerance(iterates, 5, training.COEFF, 4) * np.linalg.norm(iterates[-1]) + 3 * 2.0 ** -24 * (np.linalg.norm(w) + lr * np.linalg.norm(iterates[-1]))
    assert np.linalg.norm(W2.double().cpu().numpy() - want_W) <= tol
    gp.muon_step_tensors(W, M, G, lr, mu, wd, nesterov)     # in place
    assert same_bits(W, W2) and same_bits(M, M2)


def test_muon_steps_of_several_matrices():
    import torch
    rng = np.random.default_rng(13)
    W, M, G = (torch.from_numpy(rng.normal(size=(3, 66, 50))).float().cuda() for _ in range(3))
    alone = [gp.muon_step_tensors(W[i], M[i], G[i], 0.1, W_out=torch.empty(66, 50, device="cuda"), M_out=torch.empty(66, 50, device="cuda"))
             for i in range(3)]
    W2, M2 = gp.muon_step_tensors(W, M, G, 0.1, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    for i in range(3):
        assert same_bits(W2[i], alone[i][0]) and same_bits(M2[i], alone[i][1])


# ---- streams and graphs --------------------------------------------------------------------------------------

def all_four(s):
    gp.embedding_tensors(s["table"], s["tokens"], scale=2.0, out=s["rows"])
    gp.embedding_grad_tensors(s["tokens"], s["rows"], s["table"].shape[0], out=s["grad"], workspace=s["ws1"])
    gp.orthogonalize_tensors(s["G"], out=s["O"], workspace=s["ws2"])
    gp.muon_step_tensors(s["W"], s["M"], s["G"], 0.1, W_out=s["W2"], M_out=s["M2"], workspace=s["ws2"])


def state(N=3000, V=500, d=36):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    s = dict(table=torch.randn(V, d, generator=gen, device="cuda"), tokens=torch.randint(-1, V, (N,), generator=gen, device="cuda"),
             rows=torch.empty(N, d, device="cuda"), grad=torch.empty(V, d, device="cuda"), G=torch.randn(70, 90, generator=gen, device="cuda"),
             W=torch.randn(70, 90, generator=gen, device="cuda"), M=torch.randn(70, 90, generator=gen, device="cuda"))
    s.update(O=torch.empty_like(s["G"]), W2=torch.empty_like(s["W"]), M2=torch.empty_like(s["M"]),
             ws1=torch.empty(gp.gp_embedding_grad_workspace(N, V, d), dtype=torch.uint8, device="cuda"),
             ws2=torch.empty(gp.gp_orthogonalize_workspace(70, 90), dtype=torch.uint8, device="cuda"))
    return s


def results(s):
    return [s[k].clone() for k in ("rows", "grad", "O", "W2", "M2")]


def test_replays_of_a_captured_step():
    import torch
    s = state()
    all_four(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_four(s)
    for seed in range(4):   # other inputs in the same places, eager work and waits in between
        gen = torch.Generator(device="cuda").manual_seed(10 + seed)
        for k in ("table", "G", "W", "M"):
            s[k].copy_(torch.randn(s[k].shape, generator=gen, device="cuda"))
        s["tokens"].copy_(torch.randint(-1, 500 if seed % 2 else 4, s["tokens"].shape, generator=gen, device="cuda"))
        for k in ("rows", "grad", "O", "W2", "M2"):
            s[k].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = results(s)
        all_four(s)
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(replayed, results(s)))


def test_another_stream_than_the_current_one():
    import torch
    s = state()
    all_four(s)
    want = results(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    rows = gp.embedding_tensors(s["table"], s["tokens"], scale=2.0, stream=side.cuda_stream)
    grad = gp.embedding_grad_tensors(s["tokens"], rows, 500, stream=side.cuda_stream)
    O = gp.orthogonalize_tensors(s["G"], stream=side.cuda_stream)
    filler = [torch.full((1 << 22,), 3.0, device="cuda") for _ in range(8)]   # (the current stream's memory is others')
    side.synchronize()
    assert same_bits(rows, want[0]) and same_bits(grad, want[1]) and same_bits(O, want[2])
    del filler


@pytest.mark.parametrize("shape,count", [((64, 8192), 1), (((256, 4096)), 1), ((1000, 4097), 1), ((768, 768), 4), ((2048, 2048), 1), ((2300, 1900), 1),
                                         ((1024, 4096), 2), ((4096, 4096), 1)])
def test_orthogonalize_large(shape, count):
    """Every tile and every way to share one: against fp64 on the GPU; twice, with the same bits."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = min(shape) // 8
    G = 1e-3 * (torch.randn(count, shape[0], k, generator=gen, device="cuda") @ torch.randn(count, k, shape[1], generator=gen, device="cuda")
                + 0.2 * torch.randn(count, *shape, generator=gen, device="cuda"))
    got = gp.orthogonalize_tensors(G)
    assert same_bits(got, gp.orthogonalize_tensors(G))
    a, b, c = training.COEFF
    slope = np.abs([a + 3 * b * s ** 2 + 5 * c * s ** 4 for s in np.linspace(0.0, 1.25, 2001)]).max()
    for i in range(count):
        X = G[i].double() if shape[0] <= shape[1] else G[i].double().t().contiguous()
        X = X / (X.norm() + 1e-7)
        norms = [float(X.norm())]
        for _ in range(5):
            A = X @ X.t().contiguous()
            X = a * X + (b * A + c * (A @ A)) @ X
            norms.append(float(X.norm()))
        want = X if shape[0] <= shape[1] else X.t()
        tol = 4 * 2.0 ** -22 * sum(slope ** (5 - k) * norms[k] for k in range(6)) / norms[-1]
        assert float((got[i].double() - want).norm()) <= tol * norms[-1]


@pytest.mark.parametrize("shape", [(40, 64), (70, 200)])
@pytest.mark.parametrize("power", [-36, 36])
def test_magnitudes_at_the_ends_of_fp32(power, shape):
    """The norm's inverse, or the norm itself, lies beyond fp32's normal numbers."""
    import torch
    G = torch.from_numpy(np.random.default_rng(14).normal(size=shape) * 10.0 ** power).float().cuda()
    check_direction(gp.orthogonalize_tensors(G, eps=0.0), G, eps=0.0)


def test_one_gradient_row_for_all_tokens():
    """A gradient that was expanded from one row (rows 0 elements apart), as that of a sum is."""
    import torch
    rng = np.random.default_rng(15)
    tokens = torch.from_numpy(rng.integers(-1, 20, 500)).cuda()
    row = torch.from_numpy(rng.normal(size=(1, 37))).float().cuda()
    up = row.expand(500, 37)
    check_gradient(gp.embedding_grad_tensors(tokens, up, 20), tokens, up, 20, 1.0)


@pytest.mark.parametrize("N,V,d,tokens_kind", [(9000, 63, 5, "uniform"), (9000, 64, 5, "hot"), (20_000, 255, 3, "uniform"), (20_000, 256, 3, "uniform"),
                                               (30_000, 511, 2, "hot"), (30_000, 512, 2, "uniform"), (50_000, 2047, 1, "uniform"),
                                               (50_000, 2048, 1, "hot"), (8192, 4_300_000, 2, "uniform"), (8193, 4_194_304, 2, "uniform"),
                                               (40_000, 9_000_001, 1, "hot"), (1_300_000, 3_000_000, 3, "hot"), (1_048_577, 300, 4, "uniform")])
def test_gradient_at_the_sort_s_boundaries(N, V, d, tokens_kind):
    """Digits of 6, 8, 9 and 11 bits, one to three passes, short and long lists, small and large tiles of them."""
    import torch
    rng = np.random.default_rng(N + V)
    tokens = torch.from_numpy(tokens_of(tokens_kind, N, V, rng)).to(torch.int32).cuda()
    up = torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)).cuda()
    out = torch.full((V, d), float("nan"), device="cuda")
    gp.embedding_grad_tensors(tokens, up, V, out=out)
    check_gradient(out, tokens, up, V, 1.0)


@pytest.mark.parametrize("kind", ["low", "high", "ends", "middle"])
def test_long_gaps_between_tokens_are_zero(kind):
    """Gaps of up to 256 rows, of more, before the first token and behind the last, around every multiple of 256."""
    import torch
    V, d = 3000, 5
    places = {"low": [0, 1, 255, 256, 257], "high": [2739, 2996, 2998, 2999], "ends": [0, 2999], "middle": [1500]}[kind]
    for shift in (0, 1):
        tokens = torch.tensor([p + shift for p in places if p + shift < V], dtype=torch.int32, device="cuda").repeat(3)
        up = torch.ones(tokens.numel(), d, device="cuda")
        out = torch.full((V, d), float("nan"), device="cuda")
        gp.embedding_grad_tensors(tokens, up, V, out=out)
        want = torch.zeros(V, d, device="cuda")
        want[tokens.long()] = 3.0
        assert torch.equal(out, want)
    for gap in (255, 256, 257, 258, 511, 513):
        tokens = torch.arange(0, V, gap, dtype=torch.int32, device="cuda")
        out = torch.full((V, d), float("nan"), device="cuda")
        gp.embedding_grad_tensors(tokens, torch.ones(tokens.numel(), d, device="cuda"), V, out=out)
        want = torch.zeros(V, d, device="cuda")
        want[tokens.long()] = 1.0
        assert torch.equal(out, want)


@pytest.mark.parametrize("gap", [15, 16, 17, 31, 32, 33, 34, 63, 65, 255, 256, 257, 258])
@pytest.mark.parametrize("often", [1, 20])
def test_gaps_around_their_limits_are_zero(gap, often):
    """Few tokens for the table's rows and, each 20 times over, many: gaps of 32 and of 256 rows go either way."""
    import torch
    V, d = 2000, 6
    for first in (0, 1, gap):
        named = torch.arange(first, V, gap + 1)
        tokens = named.to(torch.int32).repeat(often).cuda()
        up = torch.ones(tokens.numel(), d, device="cuda")
        for out_dtype in (torch.float32, torch.bfloat16):
            out = torch.full((V, d), float("nan"), device="cuda", dtype=out_dtype)
            gp.embedding_grad_tensors(tokens, up, V, out=out)
            want = torch.zeros(V, d, device="cuda", dtype=out_dtype)
            want[named.cuda()] = float(often)
            assert torch.equal(out, want)


@pytest.mark.parametrize("N,V,d,low,high", [(4096, 1000, 7, 0, 1000), (4096, 32, 33, 0, 32), (4096, 31, 33, 0, 31), (4096, 1000, 3, 7, 8),
                                            (4000, 1_000_000, 4, 3906, 7812), (4000, 1_000_000, 4, 0, 3000), (129, 1000, 5, 8, 12),
                                            (128, 1000, 5, 8, 12), (1, 1, 1, 0, 1), (1, 300_000, 16, 299_999, 300_000), (3, 5, 602, 0, 5),
                                            (4096, 700, 256, 0, 700), (4096, 700, 257, 0, 700), (4097, 700, 9, 0, 700), (1025, 257, 8, 0, 257)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_of_short_lists(N, V, d, low, high, dtype):
    """Around the limits of what goes in one launch, spread over the table or all in one part of it, with tokens of no row among them."""
    import torch
    rng = np.random.default_rng(N * 31 + V + d)
    named = rng.integers(low, high, size=N)
    up = torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    for index in (torch.int32, torch.int64):
        for absent in (0.0, 0.2):
            tokens = torch.from_numpy(np.where(rng.random(N) < absent, rng.choice([-1, V, -(2 ** 31), 2 ** 31 - 1], size=N), named)).to(index).cuda()
            out = torch.full((V, d), float("nan"), device="cuda")
            gp.embedding_grad_tensors(tokens, up, V, out=out)
            check_gradient(out, tokens, up, V, 1.0)
            again = torch.empty_like(out)
            gp.embedding_grad_tensors(tokens, up, V, out=again)
            assert torch.equal(out, again)
            start = torch.from_numpy(rng.integers(-4, 5, size=(V, d)).astype(np.float32)).cuda()
            kept = start.clone()
            gp.embedding_grad_tensors(tokens, up, V, out=kept, accumulate=True)
            known = (tokens >= 0) & (tokens < V)
            rows = torch.zeros(V, dtype=torch.bool, device="cuda")
            rows[tokens[known].long()] = True
            assert torch.equal(kept[~rows], start[~rows])
            assert torch.equal(kept[rows], start[rows] + out[rows])
