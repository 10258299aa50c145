"""Layer normalisation against its formula in float64, entry by entry within bounds derived from the arithmetic."""
import pytest
import torch

from paper_2310_01655_amd import autograd
from paper_2310_01655_amd import binding as psf

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# fp32 sums of a row: at most 64 values of a lane in turn, then 8 levels of lanes and waves
NOISE = 80 * 2.0 ** -24
# and over rows: at most 20 rows of a lane in turn here, 32 lanes, 64 shares of a slice and 16 slices
ROWS_NOISE = 150 * 2.0 ** -24


def make(rows, width, dtype, seed=0, bias=True):
    g = torch.Generator().manual_seed(seed * 31 + rows + width)
    x = torch.randn(rows, width, generator=g) * (0.5 + torch.rand(rows, 1, generator=g)) + torch.randn(rows, 1, generator=g)
    w, b = 1 + 0.2 * torch.randn(width, generator=g), 0.3 * torch.randn(width, generator=g)
    dy = torch.randn(rows, width, generator=g)
    x, w, b, dy = (t.to(TYPES[dtype]).cuda() for t in (x, w, b, dy))
    return x, w, b if bias else None, dy


def reference(x, w, b, dy, eps=1e-6):
    """{name: (value, bound)}"""
    half, n = HALF_STEP[x.dtype], x.shape[1]
    x, w, dy = x.double(), w.double(), dy.double()
    mean = x.mean(1, keepdim=True)
    s = torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    u = (x - mean) / s
    # the mean is off by NOISE of the values' size, the deviation by as much relative to itself and by the mean's error squared
    em = NOISE * x.abs().mean(1, keepdim=True)
    eu = em / s + u.abs() * (2 * NOISE + (em / s) ** 2)
    y = u * w + (0 if b is None else b.double())
    g = dy * w
    c1, c2 = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    e1 = NOISE * g.abs().mean(1, keepdim=True)
    e2 = NOISE * (g * u).abs().mean(1, keepdim=True) + (g.abs() * eu).mean(1, keepdim=True)
    dx = (g - c1 - u * c2) / s
    ex = (e1 + u.abs() * e2 + eu * c2.abs() + 4 * 2.0 ** -24 * (g.abs() + c1.abs() + (u * c2).abs())) / s
    ex = ex + dx.abs() * (2 * NOISE + (em / s) ** 2)
    dw, db = (dy * u).sum(0), dy.sum(0)
    ew = (dy.abs() * eu).sum(0) + ROWS_NOISE * (dy * u).abs().sum(0)
    out = {"y": (y, eu * w.abs() + 4 * 2.0 ** -24 * (u * w).abs() + half * y.abs()),
           "dx": (dx, ex + half * dx.abs()), "dw": (dw, ew + half * dw.abs()),
           "db": (db, ROWS_NOISE * dy.abs().sum(0) + half * db.abs())}
    return out


def check(got, want, what):
    for name, t in got.items():
        if t is None:
            continue
        value, bound = want[name]
        off = (t.double() - value).abs()
        assert torch.isfinite(t).all() and (off <= 1.05 * bound + 1e-30).all(), "%s %s: %.3e over its bound" % (
            what, name, (off - bound).max())


def run(x, w, b, dy, eps=1e-6):
    y, stats = psf.psf_layer_norm_fwd(x, w, b, eps, want_stats=True)
    dx, dw, db = psf.psf_layer_norm_bwd(x, w, stats, dy, want_bias=b is not None)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 128, 129, 255, 256, 257, 512, 513, 768, 1000, 1024, 1025, 1536, 2047, 2048,
          2049, 4096, 4099, 5001, 8191, 8192]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, dtype):
    for rows in (1, 5, 67):
        x, w, b, dy = make(rows, width, dtype)
        check(run(x, w, b, dy), reference(x, w, b, dy), "%d x %d" % (rows, width))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(4999, 64), (3001, 128), (1031, 768), (2111, 37), (1500, 2056)])
def test_many_rows_without_bias(rows, width, dtype):
    x, w, _, dy = make(rows, width, dtype, seed=1, bias=False)
    check(run(x, w, None, dy), reference(x, w, None, dy), "%d x %d" % (rows, width))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_any_address(dtype):
    """Tensors that start at an element which is not a multiple of 16 bytes."""
    for width in (64, 65, 771):
        x, w, b, dy = make(50, width, dtype, seed=2)
        for shift in (1, 3):
            there = []
            for t in (x, w, b, dy):
                room = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
                room[shift:] = t.flatten()
                there.append(room[shift:].view(t.shape))
            for a, c in zip(run(x, w, b, dy).values(), run(*there).values()):
                assert torch.equal(a, c)


def test_equal_values_and_large_offsets():
    """A row of one value has deviation sqrt(eps); an offset of 1000 leaves its own rounding."""
    x = torch.full((3, 96), 7.0, device="cuda")
    one = torch.ones(96, device="cuda")
    y, stats = psf.psf_layer_norm_fwd(x, one, None, 1e-6, want_stats=True)
    assert not y.any() and (stats[:, 1] - 1000.0).abs().max() < 0.01
    x, w, b, dy = make(40, 300, "f32", seed=3)
    x += 1000.0
    check(run(x, w, b, dy), reference(x, w, b, dy), "offset")


def test_odd_rows_stay_alone():
    x, w, b, dy = make(90, 200, "bf16", seed=4)
    before = run(x, w, b, dy)
    spoilt = x.clone()
    spoilt[41, 7] = float("inf")
    spoilt[60, 0] = float("nan")
    after = run(spoilt, w, b, dy)
    keep = torch.ones(90, dtype=torch.bool, device="cuda")
    keep[[41, 60]] = False
    for name in ("y", "dx"):
        assert torch.equal(before[name][keep], after[name][keep])
        assert torch.isnan(after[name][60]).all()


def test_in_place_and_repeats():
    x, w, b, dy = make(777, 64, "bf16", seed=5)
    want = run(x, w, b, dy)
    again = run(x, w, b, dy)
    for a, c in zip(want.values(), again.values()):
        assert torch.equal(a, c)
    psf.psf_layer_norm_fwd(x, w, b, y=x)
    assert torch.equal(x, want["y"])


def test_more_than_2_31_elements():
    rows, width = 34_000_000, 64
    if torch.cuda.mem_get_info()[0] < 30 * 2 ** 30:
        pytest.skip("needs 15 GB")
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    tail, w, b, _ = make(100, width, "bf16", seed=6)
    x[-100:] = tail
    y = psf.psf_layer_norm_fwd(x, w, b)
    assert torch.equal(y[-100:], psf.psf_layer_norm_fwd(tail, w, b))


@pytest.mark.parametrize("bias", [True, False])
def test_autograd_and_graph(bias):
    x, w, b, dy = make(300, 64, "bf16", seed=7, bias=bias)
    x4 = x.view(5, 60, 64).transpose(0, 1)                     # not contiguous
    leaves = [t.detach().requires_grad_(True) for t in (x4, w, b) if t is not None]
    y = autograd.layer_norm(*leaves)
    grads = torch.autograd.grad(y, leaves, dy.view(5, 60, 64).transpose(0, 1))
    want = reference(x, w, b, dy)
    rows = lambda t: t.transpose(0, 1).reshape(300, 64)
    got = {"y": rows(y.detach()), "dx": rows(grads[0]), "dw": grads[1]}
    if bias:
        got["db"] = grads[2]
    check(got, want, "autograd")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y, stats = psf.psf_layer_norm_fwd(x, w, b, want_stats=True)
        dx, dw, db = psf.psf_layer_norm_bwd(x, w, stats, dy, want_bias=bias)
    for _ in range(3):
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        want = run(x, w, b, dy)
        for a, c in zip((y, dx, dw, db), want.values()):
            assert a is c is None or torch.equal(a, c)


def test_gradient_against_differences():
    x, w, b, dy = make(6, 40, "f32", seed=8)
    got = run(x, w, b, dy)
    g = torch.Generator().manual_seed(9)
    for name, t in (("dx", x), ("dw", w), ("db", b)):
        way, step, value = torch.randn(t.shape, generator=g).cuda(), 2.0 ** -7, []
        for sign in (1, -1):
            there = [u + sign * step * way if u is t else u for u in (x, w, b)]
            value.append((psf.psf_layer_norm_fwd(*there).double() * dy.double()).sum())
        by_difference, by_gradient = (value[0] - value[1]) / (2 * step), (got[name].double() * way.double()).sum()
        # third derivatives (step^2 / 6 of slopes of order one) and 240 roundings of 2^-24 over the step
        assert abs(by_difference - by_gradient) < 1e-2 * got[name].double().norm() + 240 * 2.0 ** -24 * 4 / step


def test_inside_the_attention_layers():
    """q_norm and k_norm are the normalisation before the call, with gradients of their parameters."""
    g = torch.Generator().manual_seed(10)
    Q, K, V, dO = (torch.randn(2, 2, 256, 64, generator=g).cuda().requires_grad_(True) for _ in range(4))
    G = torch.randn(1, psf.g_len(64, 16, 4), generator=g).cuda()
    norms = [(1 + 0.1 * torch.randn(64, generator=g)).cuda().requires_grad_(True) for _ in range(3)]
    q_norm, k_norm = (norms[0], norms[1]), (norms[2],)
    for layer in (lambda q, k, **more: autograd.causal_polysketch_attention(q, k, V, G, 4, 16, 64, **more),
                  lambda q, k, **more: autograd.causal_window_attention(q, k, V, 50, 3, **more)):
        inside = layer(Q, K, q_norm=q_norm, k_norm=k_norm)
        before = layer(autograd.layer_norm(Q, *q_norm), autograd.layer_norm(K, *k_norm))
        assert torch.equal(inside, before)
        for a, c in zip(torch.autograd.grad(inside, [Q, K, V] + norms, dO), torch.autograd.grad(before, [Q, K, V] + norms, dO)):
            assert torch.equal(a, c) and torch.isfinite(a).all() and a.any()


def test_second_derivatives_are_refused():
    x, w, b, dy = make(10, 64, "f32", seed=11)
    x.requires_grad_(True)
    y = autograd.layer_norm(x, w, b)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(y, x, dy, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        heads = x.view(1, 1, 10, 64)
        torch.autograd.grad(autograd.causal_window_attention(heads, heads, heads), x, dy.view(1, 1, 10, 64), create_graph=True)
