"""The operators around the attention layers, as cases that can be timed and compared.

  norm     layer normalisation of rows (queries and keys before an attention layer, a model's
           tokens before a block), alone or with its gradients
  window   softmax attention with a sliding window and a few first tokens that stay visible, for
           prompts (forward) and for training (output and gradients)
  paged    the same attention for one new token a sequence over a paged key-value cache
  pages    upkeep of that cache between two steps: new tokens written to their pages, sequences
           forked, the pages in use moved to the front of the pool

`run` computes them with the library where `own` is true and in elementary torch operations
where it is not; `exact` follows their definitions in float64.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ALL = 2 ** 31 - 1                                     # a window that hides nothing

_BASE = {
    "norm": dict(rows=1, width=64, dtype="bf16", bias=True, grad=False),
    "window": dict(batch=1, heads=12, kv_heads=12, n=1024, shortest=0, d=64, window=256, sinks=4, dtype="bf16",
                   tokens_first=False, grad=False),
    "paged": dict(seqs=1, heads=12, kv_heads=12, d=64, page=64, shortest=1, longest=1024, window=0, sinks=0,
                  dtype="bf16"),
    "pages": dict(seqs=64, forks=2, kv_heads=12, d=64, page=64, shortest=1, longest=1024, fresh_low=1, fresh_high=1,
                  spare=0.5, dtype="bf16"),
}


def _case(kind, **changes):
    unknown = set(changes) - set(_BASE[kind]) - {"name"}
    assert not unknown, unknown
    return {"kind": kind, **_BASE[kind], **changes}


def listed():
    return [
        # the query rows of one new token, before its attention: latency alone
        _case("norm", name="norm_token", rows=12),
        # training a GPT-2-small layer at 4k: the query rows of 8 sequences and 12 heads
        _case("norm", name="norm_heads_train", rows=8 * 12 * 4096, grad=True),
        # a numerical check of a model's tokens in fp32, sequences of odd length
        _case("norm", name="norm_model_f32_train", rows=3 * 1951, width=768, dtype="f32", grad=True),
        # a server's short prompts of unequal length, rows of a fused projection (tokens first)
        _case("window", name="window_prompts", batch=4, n=700, shortest=37, tokens_first=True),
        # training a GPT-2-small layer at 4k
        _case("window", name="window_train", batch=8, n=4096, window=1024, grad=True),
        # training at long context with wide heads, four query heads to one key head
        _case("window", name="window_train_long", batch=2, heads=16, kv_heads=4, n=16384, d=128, window=4096, grad=True),
        # a numerical check in fp32, sequences of odd and unequal length
        _case("window", name="window_train_f32", batch=2, n=1951, shortest=977, window=300, sinks=3, dtype="f32",
              grad=True),
        # one sequence being generated after a short context: latency
        _case("paged", name="paged_one", shortest=1500, longest=1500),
        # a server's batch, four query heads to one key head, contexts of unequal length
        _case("paged", name="paged_batch", seqs=64, heads=16, kv_heads=4, d=128, page=32, shortest=300, longest=12000),
        # few sequences with very long contexts: the length has to be shared out
        _case("paged", name="paged_long", seqs=3, heads=16, kv_heads=2, d=128, shortest=70001, longest=131072),
        # between two steps of a server's batch: one token each, two sequences forked, pages of ended ones reused
        _case("pages", name="pages_step", seqs=64, forks=2, kv_heads=4, d=64, page=16, longest=600),
        # a batch of prompts admitted, eight sequences forked, a pool in disorder brought together
        _case("pages", name="pages_prompts", seqs=48, forks=8, kv_heads=4, d=128, page=32, shortest=1, longest=6000,
              fresh_low=17, fresh_high=2049),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _head_size(rng):
    return rng.choice([64, 64, 64, 128, 128, 32, 80, 96, 8 * rng.randint(1, 16)])


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8, 12])
    return kv * rng.choice([1, 1, 2, 4, 5, 8]), kv


def draw(rng):
    kind = rng.choice(["norm"] * 3 + ["window"] * 5 + ["paged"] * 4 + ["pages"] * 2)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "norm":
        width = rng.choice([64, 128, 768, 1024, _log_int(rng, 1, 8192), 8 * _log_int(rng, 1, 1024)])
        return _case(kind, rows=_log_int(rng, 1, max(1, 24_000_000 // width)), width=width, dtype=dtype,
                     bias=rng.random() < 0.7, grad=rng.random() < 0.6)
    heads, kv = _heads(rng)
    d = _head_size(rng)
    if kind == "window":
        n = _log_int(rng, 1, 20000)
        case = _case(kind, batch=_log_int(rng, 1, 16), heads=heads, kv_heads=kv, n=n, d=d,
                     shortest=rng.choice([n, n, rng.randint(0, n)]),
                     window=rng.choice([_log_int(rng, 1, 8192), n, 256, 1000]), sinks=rng.choice([0, 1, 4, 4, 64, 100]),
                     dtype=dtype, tokens_first=rng.random() < 0.4, grad=rng.random() < 0.6)
        most = 5e10 if dtype == "f32" else 1.6e12
        while work(case)["flops"] > most or case["batch"] * heads * case["n"] * d > 6.6e7:
            if case["batch"] > 1:
                case["batch"] = (case["batch"] + 1) // 2
            else:
                case["n"] = case["n"] * 2 // 3
                case["shortest"] = min(case["shortest"], case["n"])
        return case
    page = rng.choice([16, 32, 64, 128, _log_int(rng, 1, 200)])
    if kind == "paged":
        longest = _log_int(rng, 1, 150000)
        case = _case(kind, seqs=_log_int(rng, 1, 128), heads=heads, kv_heads=kv, d=d, page=page,
                     shortest=rng.choice([longest, rng.randint(0, longest)]), longest=longest,
                     window=rng.choice([0, 0, _log_int(rng, 1, 8192)]), sinks=rng.choice([0, 4, 7, 64]), dtype=dtype)
        while sum(_lengths(case)) > min(2.0e8 / (kv * d * (2 if dtype == "f32" else 1)), 200_000 * page):
            if case["seqs"] > 1:
                case["seqs"] = (case["seqs"] + 1) // 2
            else:
                case["longest"] //= 2
                case["shortest"] = min(case["shortest"], case["longest"])
        return case
    seqs = _log_int(rng, 1, 128)
    longest, high = _log_int(rng, 1, 8000), _log_int(rng, 1, 2048)
    case = _case(kind, seqs=seqs, forks=rng.randint(0, min(seqs, 8)), kv_heads=kv, d=d, page=page,
                 shortest=rng.randint(0, longest), longest=longest, fresh_low=rng.randint(0, high), fresh_high=high,
                 spare=rng.uniform(0.05, 1.5), dtype=dtype)
    while _pool_tokens(case) > min(1.2e8 / (kv * d * (2 if dtype == "f32" else 1)), 200_000 * page):
        if case["seqs"] > 1:
            case["seqs"] = (case["seqs"] + 1) // 2
            case["forks"] = min(case["forks"], case["seqs"])
        else:
            case["longest"] = (case["longest"] + 1) // 2
            case["shortest"] = min(case["shortest"], case["longest"])
    return case


# ---- sizes -------------------------------------------------------------------------------

def _spread(low, high, count):
    return [high - (high - low) * i // max(1, count - 1) for i in range(count)]


def _lengths(c):
    return _spread(c["shortest"], c["longest"], c["seqs"])


def _fresh(c):
    return _spread(c["fresh_low"], c["fresh_high"], c["seqs"])


def _up(a, b):
    return -(-a // b)


def _pages_used(c):
    """Pages of the sequences with their new tokens, and one for each fork."""
    return sum(_up(a + b, c["page"]) for a, b in zip(_lengths(c), _fresh(c))) + c["forks"]


def _pool_pages(c):
    used = _pages_used(c)
    return used + max(1, int(used * c["spare"]))


def _pool_tokens(c):
    return _pool_pages(c) * c["page"]


def _window_lengths(c):
    return _spread(c["shortest"], c["n"], c["batch"])


def _pairs(n, window, sinks):
    """Visible pairs of one sequence of n tokens."""
    total = min(n, window) * (min(n, window) + 1) // 2 + max(0, n - window) * window
    beyond = max(0, n - window)                 # rows with tokens before their window: 1, 2, ... of them
    few = min(beyond, sinks)
    return total + few * (few + 1) // 2 + (beyond - few) * sinks


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "norm":
        cells = c["rows"] * c["width"]
        return {"bytes": size * cells * (5 if c["grad"] else 2), "flops": cells * (19 if c["grad"] else 8)}
    if c["kind"] == "window":
        lengths = _window_lengths(c)
        pairs = sum(_pairs(n, c["window"], c["sinks"]) for n in lengths) * c["heads"]
        cells_q, cells_k = c["batch"] * c["n"] * c["heads"] * c["d"], sum(lengths) * c["kv_heads"] * c["d"]
        if not c["grad"]:
            return {"bytes": size * (2 * cells_q + 2 * cells_k), "flops": 4 * c["d"] * pairs}
        return {"bytes": size * (4 * cells_q + 4 * cells_k), "flops": 14 * c["d"] * pairs}
    if c["kind"] == "paged":
        seen = sum(n if not c["window"] else min(n, c["window"] + c["sinks"]) for n in _lengths(c))
        return {"bytes": size * (2 * seen * c["kv_heads"] * c["d"] + 2 * c["seqs"] * c["heads"] * c["d"]),
                "flops": 4 * c["d"] * seen * c["heads"]}
    used, pages = _pages_used(c), _pool_pages(c)
    moved = used * (pages - used) / pages + c["forks"]
    token = 2 * size * c["kv_heads"] * c["d"]
    cols = _columns(c)
    return {"bytes": int(2 * token * (sum(_fresh(c)) + moved * c["page"]) + 8 * (c["seqs"] + c["forks"]) * cols),
            "flops": 0}


def _columns(c):
    if c["kind"] == "paged":
        return _up(c["longest"], c["page"]) + 1
    return _up(c["longest"] + c["fresh_high"], c["page"]) + 1


# ---- inputs ------------------------------------------------------------------------------

def _tables(c, order, rows, tokens, pool):
    """Block table [rows, columns] whose row i has the pages of tokens[i] tokens, -1 behind them."""
    table = torch.full((rows, _columns(c)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(tokens):
        need = _up(n, c["page"])
        table[i, :need] = torch.tensor(order[at:at + need], dtype=torch.int32)
        at += need
    assert at <= pool
    return table.cuda(), at


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    rng = random.Random(int(seed) * 104729 + 5)
    td = _TYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(td)

    s = {"case": c}
    if c["kind"] == "norm":
        # tokens after a projection: a common offset and a spread of their own in every row
        x = torch.randn(c["rows"], c["width"], generator=g, device="cuda")
        x = x * (0.5 + torch.rand(c["rows"], 1, generator=g, device="cuda")) + 0.3
        s["x"] = x.to(td)
        s["weight"] = (1.0 + 0.1 * torch.randn(c["width"], generator=g, device="cuda")).to(td)
        s["bias"] = (0.1 * torch.randn(c["width"], generator=g, device="cuda")).to(td) if c["bias"] else None
        if c["grad"]:
            s["dy"] = normal(c["rows"], c["width"])
            if own:
                for name in ("x", "weight", "bias"):
                    if s[name] is not None:
                        s[name].requires_grad_(True)
        return s
    if c["kind"] == "window":
        def rows(heads):
            shape = (c["batch"], c["n"], heads, c["d"]) if c["tokens_first"] else (c["batch"], heads, c["n"], c["d"])
            return normal(*shape)
        s["Q"], s["K"], s["V"] = rows(c["heads"]), rows(c["kv_heads"]), rows(c["kv_heads"])
        lengths = _window_lengths(c)
        rng.shuffle(lengths)
        s["lengths"] = None if c["shortest"] == c["n"] else torch.tensor(lengths, dtype=torch.int32).cuda()
        if c["grad"]:
            s["dO"] = rows(c["heads"])
            if own:
                for name in ("Q", "K", "V"):
                    s[name].requires_grad_(True)
        elif own:
            from paper_2310_01655_amd import binding as psf
            s["desc"] = psf.make_window_desc(c["batch"], c["heads"], c["n"], c["d"], c["window"], c["sinks"], c["dtype"],
                                             kv_heads=c["kv_heads"], tokens_first=c["tokens_first"])
        return s
    if c["kind"] == "paged":
        lengths = _lengths(c)
        rng.shuffle(lengths)
        pool = sum(_up(n, c["page"]) for n in lengths) + 3
        order = list(range(pool))
        rng.shuffle(order)
        s["table"], _ = _tables(c, order, c["seqs"], lengths, pool)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32).cuda()
        s["q"] = normal(c["seqs"], c["heads"], 1, c["d"])
        s["Kp"], s["Vp"] = (normal(pool, c["kv_heads"], c["page"], c["d"]) for _ in range(2))
        if own:
            from paper_2310_01655_amd import binding as psf
            s["desc"] = psf.make_cache_desc(pool, c["page"], c["kv_heads"], c["d"], c["seqs"], _columns(c), c["dtype"])
            s["workspace"] = psf.alloc_paged_workspace(s["desc"], c["heads"])
        return s
    lengths, fresh = _lengths(c), _fresh(c)
    rng.shuffle(lengths)
    rng.shuffle(fresh)
    pool, rows = _pool_pages(c), c["seqs"] + c["forks"]
    order = list(range(pool))
    rng.shuffle(order)
    s["table"], at = _tables(c, order, rows, [a + b for a, b in zip(lengths, fresh)], pool)
    none = [0] * c["forks"]
    s["lengths"] = torch.tensor(lengths + none, dtype=torch.int32).cuda()
    s["counts"] = torch.tensor(fresh + none, dtype=torch.int32).cuda()
    s["parents"] = torch.tensor(rng.sample(range(c["seqs"]), c["forks"]), dtype=torch.int32).cuda()
    s["children"] = torch.arange(c["seqs"], rows, dtype=torch.int32).cuda()
    s["fresh"] = torch.tensor(order[at:at + c["forks"]], dtype=torch.int32).cuda()
    n = max(1, c["fresh_high"])
    s["K"], s["V"] = (normal(rows, c["kv_heads"], n, c["d"]) for _ in range(2))
    s["Kp"], s["Vp"] = (normal(pool, c["kv_heads"], c["page"], c["d"]) for _ in range(2))
    if own:
        from paper_2310_01655_amd import binding as psf
        s["desc"] = psf.make_cache_desc(pool, c["page"], c["kv_heads"], c["d"], rows, _columns(c), c["dtype"])
        s["workspace"] = psf.alloc_compact_workspace(s["desc"])
    return s


# ---- the passes --------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, c):
    from paper_2310_01655_amd import autograd
    from paper_2310_01655_amd import binding as psf
    if c["kind"] == "norm":
        if not c["grad"]:
            return [psf.psf_layer_norm_fwd(s["x"], s["weight"], s["bias"])]
        y = autograd.layer_norm(s["x"], s["weight"], s["bias"])
        wrt = [s["x"], s["weight"]] + ([s["bias"]] if c["bias"] else [])
        return [y.detach(), *torch.autograd.grad(y, wrt, s["dy"])]
    if c["kind"] == "window":
        if not c["grad"]:
            return [psf.psf_window_attn_fwd(s["desc"], s["Q"], s["K"], s["V"], lengths=s["lengths"])]
        O = autograd.causal_window_attention(s["Q"], s["K"], s["V"], c["window"], c["sinks"], lengths=s["lengths"],
                                             tokens_first=c["tokens_first"])
        return [O.detach(), *torch.autograd.grad(O, [s["Q"], s["K"], s["V"]], s["dO"])]
    if c["kind"] == "paged":
        return [psf.psf_paged_attn(s["desc"], s["q"], s["Kp"], s["Vp"], s["table"], s["lengths"],
                                   window=c["window"] or None, sinks=c["sinks"], workspace=s["workspace"])]
    psf.psf_cache_append(s["desc"], s["K"], s["V"], s["Kp"], s["Vp"], s["table"], s["lengths"], counts=s["counts"])
    lengths = s["lengths"] + s["counts"]
    if c["forks"]:
        psf.psf_cache_fork(s["desc"], s["Kp"], s["Vp"], s["table"], lengths, s["parents"], s["children"], s["fresh"])
    table, live = psf.psf_cache_compact(s["desc"], s["Kp"], s["Vp"], s["table"], lengths, workspace=s["workspace"])
    return [s["Kp"], s["Vp"], s["table"], lengths, table, live]


def _run_plain(s, c):
    if c["kind"] == "norm":
        return _plain_norm(s, c)
    if c["kind"] == "window":
        return _plain_window(s, c)
    if c["kind"] == "paged":
        return _plain_paged(s, c)
    return _plain_pages(s, c)


def _plain_norm(s, c):
    td, n = s["x"].dtype, c["width"]
    x, w = s["x"].float(), s["weight"].float()
    centred = x - x.sum(-1, keepdim=True) / n
    inverse = 1.0 / torch.sqrt((centred * centred).sum(-1, keepdim=True) / n + 1e-6)
    unit = centred * inverse
    y = unit * w
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if not c["grad"]:
        return [y.to(td)]
    dy = s["dy"].float()
    dunit = dy * w
    dx = (dunit - dunit.sum(-1, keepdim=True) / n - unit * ((dunit * unit).sum(-1, keepdim=True) / n)) * inverse
    out = [y.to(td), dx.to(td), (dy * unit).sum(0).to(td)]
    return out + ([dy.sum(0).to(td)] if s["bias"] is not None else [])


def _plain_window(s, c):
    group, td, n = c["heads"] // c["kv_heads"], s["Q"].dtype, c["n"]
    turn = (lambda t: t.transpose(1, 2)) if c["tokens_first"] else (lambda t: t)
    Q = turn(s["Q"]).float().contiguous()
    K, V = (turn(s[x]).float().repeat_interleave(group, dim=1) for x in ("K", "V"))
    scale = 1.0 / math.sqrt(c["d"])
    O = torch.empty_like(Q)
    if c["grad"]:
        dO = turn(s["dO"]).float().contiguous()
        dQ, dK, dV = torch.empty_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    ends = torch.full((c["batch"],), n, device="cuda") if s["lengths"] is None else s["lengths"].long()
    few = min(c["sinks"], n)
    step = max(64, min(2048, int(6e8 / (c["batch"] * c["heads"] * min(n, c["window"] + few + 1024)))))
    for a in range(0, n, step):
        b = min(n, a + step)
        first = max(0, a - c["window"] + 1)
        pieces = [slice(0, b)] if first <= few else [slice(0, few), slice(first, b)]
        j = torch.cat([torch.arange(p.start, p.stop, device="cuda") for p in pieces])
        i = torch.arange(a, b, device="cuda")[:, None]
        seen = (j <= i) & ((j > i - c["window"]) | (j < c["sinks"]))
        seen = seen & (i < ends[:, None, None])                      # [batch, rows, keys]; j <= i < end
        seen = seen[:, None]
        k = torch.cat([K[:, :, p] for p in pieces], 2)
        v = torch.cat([V[:, :, p] for p in pieces], 2)
        scores = torch.matmul(Q[:, :, a:b], k.transpose(2, 3)) * scale
        scores = torch.where(seen, scores, float("-inf"))
        top = scores.amax(-1, keepdim=True)
        weights = torch.where(seen, torch.exp(scores - top), 0.0)
        total = weights.sum(-1, keepdim=True)
        weights = torch.where(total > 0, weights / total, 0.0)
        o = torch.matmul(weights, v)
        O[:, :, a:b] = o
        if c["grad"]:
            do = dO[:, :, a:b]
            dv = torch.matmul(weights.transpose(2, 3), do)
            dscores = torch.matmul(do, v.transpose(2, 3))
            dscores = weights * (dscores - (do * o).sum(-1, keepdim=True)) * scale
            dQ[:, :, a:b] = torch.matmul(dscores, k)
            dk = torch.matmul(dscores.transpose(2, 3), Q[:, :, a:b])
            at = 0
            for p in pieces:
                dK[:, :, p] += dk[:, :, at:at + p.stop - p.start]
                dV[:, :, p] += dv[:, :, at:at + p.stop - p.start]
                at += p.stop - p.start
    if not c["grad"]:
        return [turn(O.to(td)).contiguous()]
    together = lambda t: t.unflatten(1, (c["kv_heads"], group)).sum(2)
    return [turn(t.to(td)).contiguous() for t in (O, dQ, together(dK), together(dV))]


def _plain_paged(s, c):
    td, group = s["q"].dtype, c["heads"] // c["kv_heads"]
    out = torch.empty_like(s["q"])
    share = max(1, int(3e8 / (s["table"].shape[1] * c["page"] * c["kv_heads"] * c["d"])))
    for a in range(0, c["seqs"], share):
        table, ends = s["table"][a:a + share].long(), s["lengths"][a:a + share].long()
        inside = table.clamp(min=0)
        k = s["Kp"][inside].float().transpose(1, 2).flatten(2, 3)    # [seqs, kv_heads, tokens, d]
        v = s["Vp"][inside].float().transpose(1, 2).flatten(2, 3)
        q = s["q"][a:a + share].float().reshape(-1, c["kv_heads"], group, c["d"])
        j = torch.arange(k.shape[2], device="cuda")
        seen = (j < ends[:, None]) & (table >= 0).repeat_interleave(c["page"], dim=1)
        if c["window"]:
            seen = seen & ((j >= ends[:, None] - c["window"]) | (j < c["sinks"]))
        seen = seen[:, None, None]
        scores = torch.where(seen, torch.matmul(q, k.transpose(2, 3)) / math.sqrt(c["d"]), float("-inf"))
        top = scores.amax(-1, keepdim=True)
        weights = torch.where(seen, torch.exp(scores - top), 0.0)
        total = weights.sum(-1, keepdim=True)
        o = torch.where(total > 0, torch.matmul(weights, v) / total, 0.0)
        out[a:a + share] = o.reshape(-1, c["heads"], 1, c["d"]).to(td)
    return [out]


def _plain_pages(s, c):
    Kp, Vp, table, page = s["Kp"], s["Vp"], s["table"], c["page"]
    # new tokens: token t of row i goes to position lengths[i] + t
    t = torch.arange(s["K"].shape[2], device="cuda")
    row, t = (t < s["counts"][:, None]).nonzero(as_tuple=True)
    at = s["lengths"].long()[row] + t
    where, slot = table[row, at // page].long(), at % page
    Kp[where, :, slot] = s["K"][row, :, t]
    Vp[where, :, slot] = s["V"][row, :, t]
    lengths = s["lengths"] + s["counts"]
    # forks: the parent's pages, but the last one where it is not full is a copy of its own
    if c["forks"]:
        parents, children = s["parents"].long(), s["children"].long()
        ends = lengths[parents].long()
        rows = table[parents].clone()
        part = (ends % page != 0).nonzero(as_tuple=True)[0]
        last = ends[part] // page
        old = rows[part, last].long()
        rows[part, last] = s["fresh"][part]
        Kp[s["fresh"][part].long()] = Kp[old]
        Vp[s["fresh"][part].long()] = Vp[old]
        table[children] = rows
        lengths[children] = ends.int()
    # pages in use to the front: the k-th free page below their number takes the k-th used page from there on
    used = torch.arange(table.shape[1], device="cuda") * page < lengths[:, None]
    marks = torch.zeros(Kp.shape[0], dtype=torch.bool, device="cuda")
    marks[table[used].long()] = True
    live = marks.sum()
    places = torch.arange(Kp.shape[0], device="cuda")
    holes, movers = ((places < live) & ~marks).nonzero()[:, 0], ((places >= live) & marks).nonzero()[:, 0]
    Kp[holes] = Kp[movers]
    Vp[holes] = Vp[movers]
    places[movers] = holes
    moved = torch.where(used, places[table.clamp(min=0).long()].int(), -1)
    return [Kp, Vp, table, lengths, moved, live.int().reshape(1)]


# ---- from the definitions, in float64 ------------------------------------------------------

def exact(case, seed):
    c = case
    global own
    was, own = own, False                     # inputs only: no handles of the library
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "window": _exact_window, "paged": _exact_paged, "pages": _exact_pages}[c["kind"]](s, c)


def _exact_norm(s, c):
    x, w = s["x"].double(), s["weight"].double()
    bias = s["bias"].double() if c["bias"] else torch.zeros_like(w)
    deviation = torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-6)
    unit = (x - x.mean(-1, keepdim=True)) / deviation
    if not c["grad"]:
        return [unit * w + bias]
    g = s["dy"].double() * w
    dx = (g - g.mean(-1, keepdim=True) - unit * (g * unit).mean(-1, keepdim=True)) / deviation
    out = [unit * w + bias, dx, torch.einsum("rc,rc->c", s["dy"].double(), unit)]
    return out + ([s["dy"].double().sum(0)] if c["bias"] else [])


def _exact_window(s, c):
    if work(case=c)["flops"] > 6e12:
        return None
    names = ("Q", "K", "V") + (("dO",) if c["grad"] else ())
    data = {x: (s[x].transpose(1, 2) if c["tokens_first"] else s[x]).double() for x in names}
    ends = [c["n"]] * c["batch"] if s["lengths"] is None else s["lengths"].tolist()
    out = {x: torch.zeros_like(data[y]) for x, y in (("O", "Q"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"))}
    group, block = c["heads"] // c["kv_heads"], 1024
    for b, end in enumerate(ends):
        for h in range(c["heads"]):
            q, k, v = data["Q"][b, h], data["K"][b, h // group], data["V"][b, h // group]
            for lo in range(0, end, block):
                hi = min(end, lo + block)
                rows = torch.arange(lo, hi, device="cuda")
                keys = torch.arange(hi, device="cuda")
                keys = keys[(keys < c["sinks"]) | (keys > lo - c["window"])]
                ahead = rows[:, None] - keys[None, :]
                hidden = (ahead < 0) | ((ahead >= c["window"]) & (keys[None, :] >= c["sinks"]))
                logits = (q[lo:hi] @ k[keys].T) / math.sqrt(c["d"])
                p = torch.softmax(logits.masked_fill(hidden, float("-inf")), dim=1)
                out["O"][b, h, lo:hi] = p @ v[keys]
                if c["grad"]:
                    do = data["dO"][b, h, lo:hi]
                    dp = do @ v[keys].T
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(c["d"])
                    out["dQ"][b, h, lo:hi] = ds @ k[keys]
                    out["dK"][b, h // group].index_add_(0, keys, ds.T @ q[lo:hi])
                    out["dV"][b, h // group].index_add_(0, keys, p.T @ do)
    turned = {x: t.transpose(1, 2).contiguous() if c["tokens_first"] else t for x, t in out.items()}
    return [turned[x] for x in (("O", "dQ", "dK", "dV") if c["grad"] else ("O",))]


def _exact_paged(s, c):
    out = torch.zeros_like(s["q"], dtype=torch.float64)
    group = c["heads"] // c["kv_heads"]
    for i, end in enumerate(s["lengths"].tolist()):
        if end == 0:
            continue
        pages = s["table"][i, :_up(end, c["page"])].long()
        k, v = (s[x][pages].transpose(0, 1).reshape(c["kv_heads"], -1, c["d"])[:, :end].double() for x in ("Kp", "Vp"))
        if c["window"] and end > c["window"]:
            few = min(c["sinks"], end - c["window"])
            k, v = (torch.cat([x[:, :few], x[:, end - c["window"]:]], 1) for x in (k, v))
        for h in range(c["heads"]):
            logits = k[h // group] @ s["q"][i, h, 0].double() / math.sqrt(c["d"])
            out[i, h, 0] = torch.softmax(logits, 0) @ v[h // group]
    return [out]


def _exact_pages(s, c):
    page, Kp, Vp = c["page"], s["Kp"].double(), s["Vp"].double()
    table, lengths, counts = s["table"].tolist(), s["lengths"].tolist(), s["counts"].tolist()
    for i, (n, count) in enumerate(zip(lengths, counts)):
        done = 0
        while done < count:
            col, slot = divmod(n + done, page)
            take = min(page - slot, count - done)
            for pool, new in ((Kp, s["K"]), (Vp, s["V"])):
                pool[table[i][col], :, slot:slot + take] = new[i, :, done:done + take].double()
            done += take
        lengths[i] = n + count
    for parent, child, fresh in zip(s["parents"].tolist(), s["children"].tolist(), s["fresh"].tolist()):
        table[child], lengths[child] = list(table[parent]), lengths[parent]
        if lengths[parent] % page:
            col = lengths[parent] // page
            for pool in (Kp, Vp):
                pool[fresh] = pool[table[parent][col]]
            table[child][col] = fresh
    used = [row[:_up(n, page)] for row, n in zip(table, lengths)]
    marks = {p for row in used for p in row}
    live = len(marks)
    holes = [p for p in range(live) if p not in marks]
    movers = sorted(p for p in marks if p >= live)
    place = dict(zip(movers, holes))
    if movers:
        for pool in (Kp, Vp):
            pool[torch.tensor(holes)] = pool[torch.tensor(movers)]
    moved = [[place.get(p, p) for p in row] + [-1] * (len(table[0]) - len(row)) for row in used]
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return [Kp, Vp, whole(table), whole(lengths), whole(moved), whole([live])]
