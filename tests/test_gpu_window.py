"""Window attention (forward, backward, autograd) against its definition in float64, entry by entry within
bounds derived from the arithmetic (window_reference.py)."""
import pytest
import torch

from paper_2310_01655_amd import autograd
from paper_2310_01655_amd import binding as psf
from window_reference import assert_within, window_reference

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(batch, heads, kv, n, d, dtype, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed * 1009 + n + d)
    rows = lambda h, x=1.0: (x * torch.randn(batch, h, n, d, generator=g)).to(TYPES[dtype]).cuda()
    return rows(heads, spread), rows(kv), rows(kv), rows(heads)


def run(Q, K, V, dO, window, sinks, lengths=None, scale=None, tokens_first=False):
    turn = (lambda t: t.transpose(1, 2).contiguous()) if tokens_first else (lambda t: t)
    back = (lambda t: t.transpose(1, 2)) if tokens_first else (lambda t: t)
    batch, heads, n, d = Q.shape
    desc = psf.make_window_desc(batch, heads, n, d, window, sinks, psf.BF16 if Q.dtype == torch.bfloat16 else psf.F32,
                                kv_heads=K.shape[1], tokens_first=tokens_first, scale=scale)
    q, k, v, g = (turn(t) for t in (Q, K, V, dO))
    O, lse = psf.psf_window_attn_fwd(desc, q, k, v, lengths=lengths, want_lse=True)
    grads = psf.psf_window_attn_bwd(desc, q, k, v, O, lse, g, lengths=lengths)
    return dict(zip(("O", "dQ", "dK", "dV"), (back(t) for t in (O, *grads)))), lse


def check(got, want, what):
    for name, (value, bound) in want.items():
        assert_within(got[name], value, bound, "%s %s" % (what, name))


SHAPES = [
    # batch, heads, kv, n, d, window, sinks
    (1, 1, 1, 1, 64, 1, 0), (1, 1, 1, 2, 64, 1, 0), (2, 3, 3, 31, 64, 4, 1), (1, 2, 1, 33, 64, 100, 0),
    (1, 2, 2, 64, 64, 64, 0), (1, 1, 1, 65, 64, 32, 65), (2, 4, 2, 127, 64, 1, 3), (1, 2, 2, 129, 64, 16, 4),
    (1, 6, 2, 200, 64, 50, 33), (1, 2, 2, 257, 64, 256, 4), (1, 2, 1, 400, 128, 100, 4), (2, 4, 1, 300, 128, 64, 70),
    (1, 2, 2, 191, 8, 40, 2), (1, 2, 2, 150, 32, 40, 2), (1, 2, 2, 190, 72, 60, 9), (1, 2, 2, 140, 80, 140, 0),
    (1, 1, 1, 260, 96, 33, 1), (1, 5, 1, 130, 120, 70, 4), (1, 1, 1, 700, 64, 700, 0), (1, 1, 1, 900, 64, 130, 129),
    (1, 16, 2, 330, 128, 200, 5), (3, 2, 2, 513, 64, 65, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_and_gradients(shape, dtype):
    batch, heads, kv, n, d, window, sinks = shape
    Q, K, V, dO = make(batch, heads, kv, n, d, dtype)
    got, _ = run(Q, K, V, dO, window, sinks)
    check(got, window_reference(Q, K, V, window, sinks, dO=dO), str(shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape,lengths", [
    ((3, 2, 1, 200, 64, 50, 4), (0, 1, 200)), ((4, 2, 2, 130, 128, 40, 0), (64, 65, 129, 300)),
    ((3, 4, 2, 300, 64, 299, 3), (-5, 128, 257)),
])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_unequal_lengths(shape, lengths, dtype, tokens_first):
    """Rows behind a length are not read (they hold NaN) and come back as zeros."""
    batch, heads, kv, n, d, window, sinks = shape
    Q, K, V, dO = make(batch, heads, kv, n, d, dtype, seed=1)
    want = window_reference(Q, K, V, window, sinks, lengths=lengths, dO=dO)
    for b, end in enumerate(lengths):
        for t in (Q, K, V, dO):
            t[b, :, max(end, 0):] = float("nan")
    got, lse = run(Q, K, V, dO, window, sinks, torch.tensor(lengths, dtype=torch.int32).cuda(), tokens_first=tokens_first)
    check(got, want, str(shape))
    for b, end in enumerate(lengths):
        for t in got.values():
            assert not t[b, :, max(end, 0):].any()
        assert (lse[b, :, max(end, 0):] == float("-inf")).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_first_and_scale(dtype):
    Q, K, V, dO = make(2, 6, 2, 210, 64, dtype, seed=2)
    for scale in (0.3, -0.2, 0.0):
        got, _ = run(Q, K, V, dO, 77, 5, scale=scale, tokens_first=True)
        check(got, window_reference(Q, K, V, 77, 5, scale=scale, dO=dO), "tokens first, scale %g" % scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0])
def test_score_sizes(dtype, spread):
    """Equal weights, nearly equal ones, and weights of which one is all (the maximum moves from tile to tile)."""
    Q, K, V, dO = make(1, 2, 2, 300, 64, dtype, seed=3, spread=spread)
    got, _ = run(Q, K, V, dO, 170, 4)
    check(got, window_reference(Q, K, V, 170, 4, dO=dO), "spread %g" % spread)


def test_growing_scores():
    """Scores that rise along the sequence by hundreds: every tile brings a new maximum."""
    Q, K, V, dO = make(1, 1, 1, 320, 64, "bf16", seed=4)
    K *= torch.linspace(0, 20, 320, device="cuda")[:, None].to(K.dtype)
    K.copy_(torch.where(torch.arange(320, device="cuda")[:, None] % 3 == 0, Q[0, 0, -1] * K[0, 0, :, :1].abs(), K))
    got, _ = run(Q, K, V, dO, 320, 0)
    check(got, window_reference(Q, K, V, 320, 0, dO=dO), "growing")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(2, 3, 3, 40, 64), (1, 4, 2, 130, 120), (1, 2, 1, 300, 128)])
def test_rows_of_one_key_have_no_score_gradient(shape, dtype):
    """With a window of one token p = 1 and dS = p (<dO, v> - D) = 0, whatever o was rounded to.  What may stay: p is
    exp2 of a sum of a few fp32 roundings of |L| < 64 (2^-16 relative), and <dO, v> itself of d terms in two orders
    (2^-16 of the sum of its terms' sizes at d = 128)."""
    Q, K, V, dO = make(*shape, dtype, seed=11)
    got, lse = run(Q, K, V, dO, window=1, sinks=0)
    assert lse.abs().max() < 64
    wide = lambda t: t.double().repeat_interleave(shape[1] // shape[2], 1) if t.shape[1] != shape[1] else t.double()
    q, k, v, g = (wide(t) for t in (Q, K, V, dO))
    left = (g.abs() * v.abs()).sum(-1, keepdim=True) * 2.0 ** -15 / shape[4] ** 0.5
    assert (got["dQ"].double().abs() <= left * k.abs()).all()
    most = (left * q.abs()).reshape(shape[0], shape[2], -1, *q.shape[2:]).sum(2)
    assert (got["dK"].double().abs() <= most).all()


@pytest.mark.parametrize("shape,lengths", [
    ((1, 1, 1, 1, 64, 1, 0), None), ((2, 4, 2, 7, 48, 3, 1), [7, 0]), ((3, 8, 2, 32, 128, 40, 0), [32, 5, 31]), ((1, 2, 1, 31, 8, 2, 4), None),
])
def test_short_calls_round_the_results_only(shape, lengths):
    """Up to 32 tokens in bf16 storage: the bounds of fp32 storage and one rounding of the result (2^-8, half a step)."""
    Q, K, V, dO = make(*shape[:5], "bf16", seed=12)
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got, _ = run(Q, K, V, dO, *shape[5:], lengths=ends)
    want = window_reference(*(t.float() for t in (Q, K, V)), *shape[5:], lengths=lengths, dO=dO.float())
    check(got, {x: (value, bound * (1 + 2.0 ** -8) + 2.0 ** -8 * value.abs()) for x, (value, bound) in want.items()}, "short")


def test_lse():
    Q, K, V, dO = make(2, 4, 2, 150, 64, "f32", seed=5)
    _, lse = run(Q, K, V, dO, 40, 3)
    for b in range(2):
        for h in range(4):
            s = (Q[b, h].double() @ K[b, h // 2].double().T) / 8
            i, j = torch.arange(150, device="cuda")[:, None], torch.arange(150, device="cuda")[None]
            s = torch.where((j <= i) & ((i - j < 40) | (j < 3)), s, float("-inf"))
            # score errors (64 + 8) 2^-23 of sums below 12, the logarithm's own, one rounding
            assert (lse[b, h].double() - s.logsumexp(1)).abs().max() < 72 * 2.0 ** -23 * 12 + 2.0 ** -20


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,at", [(200, 97), (60, 31)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_odd_values_stay_with_the_rows_that_see_them(dtype, d, value, n, at):
    """A non-finite K, V, Q or dO row changes nothing for tokens that share no visible pair with it."""
    window, sinks = 20, 3
    Q, K, V, dO = make(1, 2, 2, n, d, dtype, seed=6)
    before, _ = run(Q, K, V, dO, window, sinks)
    rows = torch.arange(n, device="cuda")
    sees = (rows >= at) & (rows - at < window)                     # rows that see token `at`
    seen = (rows <= at) & ((at - rows < window) | (rows < sinks))   # tokens that row `at` sees
    near = torch.zeros(n, dtype=torch.bool, device="cuda")          # tokens that share a row with token `at`
    for i in range(at, min(n, at + window)):
        near |= (rows <= i) & ((i - rows < window) | (rows < sinks))
    for name, spoilt in (("V", {"O": sees, "dQ": sees, "dK": near, "dV": near}),
                         ("K", {"O": sees, "dQ": sees, "dK": near, "dV": near}),
                         ("Q", {"O": rows == at, "dQ": rows == at, "dK": seen, "dV": seen}),
                         ("dO", {"O": rows < 0, "dQ": rows == at, "dK": seen, "dV": seen})):
        tensors = {"Q": Q.clone(), "K": K.clone(), "V": V.clone(), "dO": dO.clone()}
        tensors[name][0, 0, at, 5] = value
        after, _ = run(*(tensors[x] for x in ("Q", "K", "V", "dO")), window, sinks)
        for out, mask in spoilt.items():
            assert torch.isfinite(after[out][0, 1]).all() and torch.equal(after[out][0, 1], before[out][0, 1])
            keep = ~mask
            assert torch.isfinite(after[out][0, 0][keep]).all(), (name, out)
            # (a tile that holds such a value may be summed in another order)
            scale = before[out][0, 0].double().abs().max()
            step = 4 * 2.0 ** -8 if dtype == "bf16" else 64 * 2.0 ** -24
            assert (after[out][0, 0][keep].double() - before[out][0, 0][keep].double()).abs().max() <= step * scale, (name, out)
    tensors = {"V": V.clone()}
    tensors["V"][0, 0, at, 5] = value
    after, _ = run(Q, K, tensors["V"], dO, window, sinks)
    got = after["O"][0, 0, :, 5][sees].double()
    assert (torch.isnan(got) if value != value else got == value).all()


def test_repeated_calls_and_streams_and_graph():
    Q, K, V, dO = make(2, 4, 2, 500, 64, "bf16", seed=7)
    first, _ = run(Q, K, V, dO, 90, 70)
    other = torch.cuda.Stream()
    desc = psf.make_window_desc(2, 4, 500, 64, 90, 70, kv_heads=2)
    other.wait_stream(torch.cuda.current_stream())
    O, lse = psf.psf_window_attn_fwd(desc, Q, K, V, want_lse=True, stream=other)
    grads = psf.psf_window_attn_bwd(desc, Q, K, V, O, lse, dO, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    for a, b in zip(first.values(), (O, *grads)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        O, lse = psf.psf_window_attn_fwd(desc, Q, K, V, want_lse=True)
        grads = psf.psf_window_attn_bwd(desc, Q, K, V, O, lse, dO)
    for k in range(3):
        V.copy_(torch.roll(V, 1, 2))
        graph.replay()
        torch.cuda.synchronize()
        want, _ = run(Q, K, V, dO, 90, 70)
        torch.cuda.synchronize()
        for a, b in zip(want.values(), (O, *grads)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("tokens_first", [False, True])
def test_autograd(tokens_first):
    """Through torch.autograd, with leaves that are views (not contiguous) and a gradient that is one."""
    g = torch.Generator().manual_seed(9)
    shape = (2, 90, 4, 64) if tokens_first else (2, 4, 90, 64)
    Q, K, V, dO = (torch.randn(*shape[:3], 128, generator=g).cuda()[..., ::2].detach().requires_grad_(True) for _ in range(4))
    lengths = torch.tensor([90, 41], dtype=torch.int32).cuda()
    O = autograd.causal_window_attention(Q, K, V, 30, 2, lengths=lengths, tokens_first=tokens_first)
    grads = torch.autograd.grad(O, (Q, K, V), dO)
    turn = (lambda t: t.detach().transpose(1, 2)) if tokens_first else (lambda t: t.detach())
    want = window_reference(turn(Q), turn(K), turn(V), 30, 2, lengths=[90, 41], dO=turn(dO))
    check({x: turn(t) for x, t in zip(("O", "dQ", "dK", "dV"), (O, *grads))}, want, "autograd")


def test_gradient_against_differences():
    """Directional derivatives of sum(O * dO) in fp32 storage against central differences of the forward call."""
    Q, K, V, dO = make(1, 2, 1, 70, 32, "f32", seed=10)
    got, _ = run(Q, K, V, dO, 20, 2)
    g = torch.Generator().manual_seed(11)
    for name, x in (("dQ", Q), ("dK", K), ("dV", V)):
        way = torch.randn(x.shape, generator=g).cuda()
        step = 2.0 ** -7
        value = []
        for sign in (1, -1):
            there = {"dQ": Q, "dK": K, "dV": V}
            there = {k: (t + sign * step * way if k == name else t) for k, t in there.items()}
            out, _ = run(there["dQ"], there["dK"], there["dV"], dO, 20, 2)
            value.append((out["O"].double() * dO.double()).sum())
        by_difference = (value[0] - value[1]) / (2 * step)
        by_gradient = (got[name].double() * way.double()).sum()
        # third derivative step^2 / 6 of a function with slopes of order |gradient|, and rounding 2^-24 of 4480 terms / step
        assert abs(by_difference - by_gradient) < 1e-2 * got[name].double().norm() + 4480 * 2.0 ** -24 / step


def test_long_offsets():
    """Heads whose rows lie beyond 2^31 elements of the tensor."""
    n, d, heads = 70000, 128, 250
    if torch.cuda.mem_get_info()[0] < 40 * 2 ** 30:
        pytest.skip("needs 20 GB")
    Q = torch.zeros(1, heads, n, d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.zeros(1, heads, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(12)
    for t in (Q, K, V):
        t[0, -1, -200:] = torch.randn(200, d, generator=g).cuda()
    desc = psf.make_window_desc(1, heads, n, d, 150, 0)
    O = psf.psf_window_attn_fwd(desc, Q, K, V)
    want = window_reference(*(t[:, -1:, -200:].clone() for t in (Q, K, V)), 150, 0)["O"]
    assert_within(O[:, -1:, -50:], want[0][:, :, -50:], want[1][:, :, -50:], "last rows")
