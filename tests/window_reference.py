"""Window attention from its definition in float64, pair by pair, with an error bound for every output
(test infrastructure).

The bounds follow the arithmetic of a correct implementation on the stored inputs; u is half a step of the storage
type relative to a value (bf16 2^-8, fp32 2^-24), r the rounding of a weight for its product (2^-8 in bf16
storage, 2^-22 for fp32 from three parts), all first order with a few per cent on top:
  score     |error| <= ds = |scale| (d + 8) 2^-23 sum_c |q_c k_c|       (fp32 products and sums)
  weight    relative error E <= 2 max_j ds + (4 + max |s|) 2^-21      (exponent, maximum, sum, L)
  o         sum_j p (r + E + (n + 8) 2^-24) |v| + u |o|
  D         sum_c |dO_c| (error of the stored o_c + (d + 8) 2^-24 |o_c|)
  dS        p (r |t| + E |t| + eD + e_t),  t = <dO, v> - D,  e_t = (d + 8) 2^-23 sum_c |dO_c v_c|
  dQ, dK    |scale| sum (error of dS + (n + 8) 2^-24 |dS|) |k or q| + u |result|
  dV        sum_i p (r + E + (n + 8) 2^-24) |dO| + u |dV|
"""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
WEIGHT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -22}


def visible(n, end, window, sinks, device):
    i, j = torch.arange(n, device=device)[:, None], torch.arange(n, device=device)[None]
    return (j <= i) & ((i - j < window) | (j < sinks)) & (i < end)


def window_reference(Q, K, V, window, sinks, lengths=None, scale=None, dO=None):
    """Q, dO [batch, heads, n, d], K, V [batch, kv_heads, n, d]; returns {name: (value, bound)} in float64."""
    batch, heads, n, d = Q.shape
    group, u, r = heads // K.shape[1], HALF_STEP[Q.dtype], WEIGHT[Q.dtype]
    scale = d ** -0.5 if scale is None else scale
    names = ("O",) + (("dQ", "dK", "dV") if dO is not None else ())
    like = {"O": Q, "dQ": Q, "dK": K, "dV": V}
    out = {x: (torch.zeros_like(like[x], dtype=torch.float64), torch.zeros_like(like[x], dtype=torch.float64)) for x in names}
    sums = (n + 8) * 2.0 ** -24
    for b in range(batch):
        end = n if lengths is None else min(max(int(lengths[b]), 0), n)
        seen = visible(n, end, window, sinks, Q.device)[:end, :end]
        if end == 0:
            continue
        for h in range(heads):
            kv = h // group
            q, k, v = Q[b, h, :end].double(), K[b, kv, :end].double(), V[b, kv, :end].double()
            s = torch.where(seen, scale * (q @ k.T), float("-inf"))
            p = torch.softmax(s, 1)
            ds = torch.where(seen, abs(scale) * (d + 8) * 2.0 ** -23 * (q.abs() @ k.abs().T), 0.0)
            E = 2 * ds.amax(1, keepdim=True) + (4 + torch.where(seen, s.abs(), 0.0).amax(1, keepdim=True)) * 2.0 ** -21
            o = p @ v
            bound = (p * (r + E + sums)) @ v.abs() + u * o.abs()
            out["O"][0][b, h, :end], out["O"][1][b, h, :end] = o, bound
            if dO is None:
                continue
            g = dO[b, h, :end].double()
            D = (g * o).sum(1, keepdim=True)
            eD = (g.abs() * (bound + (d + 8) * 2.0 ** -24 * o.abs())).sum(1, keepdim=True)
            t = g @ v.T - D
            et = (d + 8) * 2.0 ** -23 * (g.abs() @ v.abs().T)
            dS = p * t
            eS = p * ((r + E) * t.abs() + eD + et) + sums * dS.abs()
            out["dQ"][0][b, h, :end] = scale * (dS @ k)
            out["dQ"][1][b, h, :end] = abs(scale) * (eS @ k.abs())
            out["dK"][0][b, kv, :end] += scale * (dS.T @ q)
            out["dK"][1][b, kv, :end] += abs(scale) * (eS.T @ q.abs())
            out["dV"][0][b, kv, :end] += p.T @ g
            out["dV"][1][b, kv, :end] += (p * (r + E + sums)).T @ g.abs()
    for x in names[1:]:
        out[x][1].add_(u * out[x][0].abs())
    return out


def assert_within(got, want, bound, what=""):
    """Every entry within its bound (5 per cent for second order terms)."""
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - want).abs()
    over = off - 1.05 * bound - 1e-30
    at = over.argmax()
    assert (over <= 0).all(), "%s: off by %.3e at %s, bound %.3e, value %.3e" % (
        what, off.flatten()[at], [int(x) for x in torch.unravel_index(at, off.shape)], bound.flatten()[at], want.flatten()[at])
