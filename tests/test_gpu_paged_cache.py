"""The paged cache: appending, forking and compacting against a plain model of it (equal bit for bit), and attention of
one new token over it against the definition in float64."""
import random

import pytest
import torch

from paper_2310_01655_amd import autograd
from paper_2310_01655_amd import binding as psf
from window_reference import HALF_STEP, WEIGHT, assert_within

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def make_cache(lengths, page, kv, d, dtype, seed=0, spare=5, cols=None):
    """Pools of normal values, a table of pages in random order; free pages and unused slots hold NaN."""
    rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + spare
    order = list(range(pages))
    rng.shuffle(order)
    cols = max(need + [1]) + 1 if cols is None else cols
    table = torch.full((len(lengths), cols), -1, dtype=torch.int32)
    Kp, Vp = (torch.full((pages, kv, page, d), float("nan")).to(TYPES[dtype]) for _ in range(2))
    at = 0
    for i, n in enumerate(lengths):
        for c in range(need[i]):
            p = order[at]
            at += 1
            if c < cols:
                table[i, c] = p
            used = min(page, n - c * page)
            for pool in (Kp, Vp):
                pool[p, :, :used] = torch.randn(kv, used, d, generator=g).to(TYPES[dtype])
    desc = psf.make_cache_desc(pages, page, kv, d, len(lengths), cols, dtype)
    return desc, Kp.cuda(), Vp.cuda(), table.cuda(), ints(lengths), order[at:]


def dense(pool, table, i, n, page):
    """Rows of sequence i ([kv, n, d], float64) and which of them lie on a page of the pool."""
    rows = [int(table[i, t // page]) if t // page < table.shape[1] else -1 for t in range(0, n, page)]
    there = torch.tensor([0 <= p < pool.shape[0] for p in rows for _ in range(page)][:n], dtype=torch.bool)
    safe = torch.tensor([p if 0 <= p < pool.shape[0] else 0 for p in rows]).cuda()
    return pool[safe].transpose(0, 1).flatten(1, 2)[:, :n].double(), there.cuda()


def reference(q, Kp, Vp, table, lengths, page, window=None, sinks=0, scale=None):
    seqs, heads, _, d = q.shape
    group, u, r = heads // Kp.shape[1], HALF_STEP[q.dtype], WEIGHT[q.dtype]
    scale = d ** -0.5 if scale is None else scale
    out, bound = torch.zeros_like(q, dtype=torch.float64), torch.zeros_like(q, dtype=torch.float64)
    for i in range(seqs):
        n = max(int(lengths[i]), 0)
        if n == 0:
            continue
        k, there = dense(Kp, table, i, n, page)
        v, _ = dense(Vp, table, i, n, page)
        j = torch.arange(n, device="cuda")
        seen = there & ((n - 1 - j < (n if window is None else window)) | (j < sinks))
        if not seen.any():
            continue
        for h in range(heads):
            kk, vv, qq = k[h // group][seen], v[h // group][seen], q[i, h, 0].double()
            s = scale * (kk @ qq)
            p = torch.softmax(s, 0)
            ds = scale * (d + 8) * 2.0 ** -23 * (kk.abs() @ qq.abs())
            E = 2 * ds.max() + (4 + s.abs().max()) * 2.0 ** -21
            out[i, h, 0] = p @ vv
            # (sums: 32 products in turn a step, steps of a wave in turn, then waves and splits)
            bound[i, h, 0] = (p * (r + E + (len(p) / 16 + 64) * 2.0 ** -24)) @ vv.abs() + u * out[i, h, 0].abs()
    return out, bound


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,page,heads,kv,d,window,sinks", [
    ((1,), 16, 1, 1, 64, None, 0), ((0, 1, 2, 31, 32, 33), 16, 4, 2, 64, None, 0), ((300, 299, 0, 1000), 32, 8, 2, 128, None, 0),
    ((70, 129), 1, 2, 2, 64, None, 0), ((200, 75), 7, 3, 1, 64, 50, 3), ((500, 40, 64), 48, 16, 1, 128, 100, 40),
    ((400,), 128, 17, 1, 64, 1, 0), ((333, 90), 64, 40, 2, 64, 64, 70), ((150, 151), 16, 4, 4, 8, None, 0),
    ((260, 10), 20, 6, 3, 72, 33, 4), ((260,), 256, 5, 5, 96, 200, 1), ((100, 65), 16, 20, 4, 120, None, 0),
    ((5000,), 64, 4, 1, 64, 1000, 4), ((3000, 7000), 32, 12, 12, 64, None, 0),
])
def test_attention_of_one_token(lengths, page, heads, kv, d, window, sinks, dtype):
    desc, Kp, Vp, table, n, _ = make_cache(lengths, page, kv, d, dtype, seed=len(lengths) + page)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(len(lengths), heads, 1, d, generator=g).to(TYPES[dtype]).cuda()
    o = psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=window, sinks=sinks)
    assert_within(o, *reference(q, Kp, Vp, table, lengths, page, window, sinks), what=str((lengths, page)))
    for i, length in enumerate(lengths):
        if length == 0:
            assert not o[i].any()
    assert torch.equal(o, psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=window, sinks=sinks))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_table_for_short_sequences(dtype):
    """The splits go by what the table can hold; sequences far shorter than that leave most of them empty."""
    desc, Kp, Vp, table, n, _ = make_cache((1, 33, 0, 700), 16, 2, 64, dtype, seed=5, cols=5000)
    q = torch.randn(4, 4, 1, 64, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).cuda()
    assert psf.paged_workspace_bytes(desc, 4) > 0
    o = psf.psf_paged_attn(desc, q, Kp, Vp, table, n, scale=0.5)
    assert_within(o, *reference(q, Kp, Vp, table, (1, 33, 0, 700), 16, scale=0.5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_freed_and_bad_pages_are_not_seen(dtype):
    """Entries outside the pool stand for no page, wherever they are; a table shorter than a length ends it."""
    lengths, page = [200, 130, 90], 16
    desc, Kp, Vp, table, n, _ = make_cache(lengths, page, 2, 64, dtype, seed=7)
    q = torch.randn(3, 4, 1, 64, generator=torch.Generator().manual_seed(8)).to(TYPES[dtype]).cuda()
    table[0, 1:6] = -1                                         # between the first tokens and the window
    table[1, 2], table[1, 3] = desc.pages, 2 ** 31 - 1
    table[2, :] = -7
    for window, sinks in ((None, 0), (60, 4), (3, 0)):
        o = psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=window, sinks=sinks)
        assert_within(o, *reference(q, Kp, Vp, table, lengths, page, window, sinks))
        assert not o[2].any()
    short = table[:, :5].contiguous()
    desc5 = psf.make_cache_desc(desc.pages, page, 2, 64, 3, 5, dtype)
    o = psf.psf_paged_attn(desc5, q, Kp, Vp, short, n)
    assert_within(o, *reference(q, Kp, Vp, short, lengths, page))
    o = psf.psf_paged_attn(desc, q, Kp, Vp, table, ints([-3, -2 ** 31, 0]))
    assert not o.any()


def test_odd_values_of_one_sequence():
    lengths, page = (100, 200), 16
    desc, Kp, Vp, table, n, _ = make_cache(lengths, page, 2, 64, "bf16", seed=9)
    q = torch.randn(2, 4, 1, 64, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    before = psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=50)
    Vp[int(table[0, 0])], Kp[int(table[0, 1])] = float("nan"), float("inf")          # outside the window
    assert torch.equal(before, psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=50))
    Vp[int(table[0, 5]), 0, 10, 3] = float("inf")                                  # position 90
    after = psf.psf_paged_attn(desc, q, Kp, Vp, table, n, window=50)
    assert (after[0, :2, 0, 3] == float("inf")).all() and torch.equal(before[:, 2:], after[:, 2:])
    assert torch.equal(before[1], after[1])


def test_positions_beyond_2_31_elements():
    page, kv, d, pages = 64, 4, 128, 70000
    if torch.cuda.mem_get_info()[0] < 24 * 2 ** 30:
        pytest.skip("needs 10 GB")
    Kp, Vp = (torch.zeros(pages, kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    for pool in (Kp, Vp):
        pool[-2:] = torch.randn(2, kv, page, d, generator=g).cuda()
    desc = psf.make_cache_desc(pages, page, kv, d, 1, 3)
    table, q = ints([[pages - 1, pages - 2, -1]]), torch.randn(1, 8, 1, d, generator=g).to(torch.bfloat16).cuda()
    o = psf.psf_paged_attn(desc, q, Kp, Vp, table, ints([100]))
    assert_within(o, *reference(q, Kp, Vp, table, [100], page))
    new = torch.randn(1, kv, 20, d, generator=g).to(torch.bfloat16).cuda()
    psf.psf_cache_append(desc, new, -new, Kp, Vp, table, ints([100]))
    assert torch.equal(Kp[pages - 2, :, 36:56], new[0]) and torch.equal(Vp[pages - 2, :, 36:56], -new[0])


# ---- upkeep ------------------------------------------------------------------------------------

def model_append(K, V, Kp, Vp, table, lengths, counts, page):
    for i, (n, count) in enumerate(zip(lengths, counts)):
        for t in range(min(count, K.shape[2]) if n >= 0 else 0):
            c, s = divmod(n + t, page)
            if c < table.shape[1] and 0 <= int(table[i, c]) < Kp.shape[0]:
                Kp[int(table[i, c]), :, s], Vp[int(table[i, c]), :, s] = K[i, :, t], V[i, :, t]


def same(a, b):
    return torch.equal(a.view(torch.int16 if a.element_size() == 2 else torch.int32),
                       b.view(torch.int16 if b.element_size() == 2 else torch.int32))      # NaN included


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,counts,page,kv,d,n", [
    ((0,), (1,), 16, 1, 64, 1), ((0, 15, 16, 31), (1, 1, 1, 1), 16, 2, 64, 1), ((3, 100, 0), (0, 33, 40), 8, 3, 72, 40),
    ((5, 5), (300, 7), 64, 2, 128, 300), ((10, 0, 2), (9, 99, 3), 5, 1, 8, 9), ((20,) * 40, (1,) * 40, 7, 4, 24, 1),
])
def test_append(lengths, counts, page, kv, d, n, dtype):
    desc, Kp, Vp, table, have, _ = make_cache([a + min(c, n) for a, c in zip(lengths, counts)], page, kv, d, dtype)
    g = torch.Generator().manual_seed(2)
    K, V = (torch.randn(len(lengths), kv, n, d, generator=g).to(TYPES[dtype]) for _ in range(2))
    want_k, want_v = Kp.cpu(), Vp.cpu()
    model_append(K, V, want_k, want_v, table.cpu(), lengths, counts, page)
    psf.psf_cache_append(desc, K.cuda(), V.cuda(), Kp, Vp, table, ints(lengths), counts=ints(counts))
    assert same(Kp.cpu(), want_k) and same(Vp.cpu(), want_v)
    if all(c == n for c in counts):
        Kp2, Vp2 = torch.zeros_like(Kp), torch.zeros_like(Vp)
        psf.psf_cache_append(desc, K.cuda(), V.cuda(), Kp2, Vp2, table, ints(lengths))
        assert Kp2.any() and same(torch.where(Kp2 != 0, Kp, Kp2), Kp2)


def test_append_leaves_out_what_has_no_place():
    desc, Kp, Vp, table, _, _ = make_cache((40, 40, 40), 16, 2, 64, "bf16")
    table[1, 1], table[2, 0] = -1, 10 ** 6
    K = torch.ones(3, 2, 30, 64, dtype=torch.bfloat16)
    want_k, want_v = Kp.cpu(), Vp.cpu()
    model_append(K, K, want_k, want_v, table.cpu(), (60, 10, 5), (30, 30, 30), 16)
    psf.psf_cache_append(desc, K.cuda(), K.cuda(), Kp, Vp, table, ints((60, 10, 5)), counts=ints((30, 99, 30)))
    assert same(Kp.cpu(), want_k) and same(Vp.cpu(), want_v)
    psf.psf_cache_append(desc, K.cuda(), K.cuda(), Kp, Vp, table, ints((-1, 2 ** 31 - 1, -2 ** 31)))
    psf.psf_cache_append(desc, K.cuda(), K.cuda(), Kp, Vp, table, ints((0, 0, 0)), counts=ints((0, -4, 0)))
    assert same(Kp.cpu(), want_k) and same(Vp.cpu(), want_v)


@pytest.mark.parametrize("dtype,page,kv,d", [("bf16", 16, 2, 64), ("f32", 7, 3, 8), ("bf16", 64, 8, 128)])
def test_fork(dtype, page, kv, d):
    lengths = [5 * page + 3, 4 * page, 0, 1, 0, 0, 0, 0, 0]
    desc, Kp, Vp, table, n, free = make_cache(lengths, page, kv, d, dtype, spare=9)
    parents, children, fresh = [0, 1, 0, 3, 2, 99, 1], [4, 5, 6, 7, 8, 4, -1], free[:7]
    want_k, want_v, rows, ends = Kp.cpu(), Vp.cpu(), table.cpu(), list(lengths)
    for a, b, f in zip(parents, children, fresh):
        if not (0 <= a < 9 and 0 <= b < 9):
            continue
        rows[b], ends[b] = rows[a], ends[a]
        if ends[a] % page:
            old = int(rows[a, ends[a] // page])
            rows[b, ends[a] // page] = f
            want_k[f], want_v[f] = want_k[old], want_v[old]
    psf.psf_cache_fork(desc, Kp, Vp, table, n, ints(parents), ints(children), ints(fresh))
    assert same(Kp.cpu(), want_k) and same(Vp.cpu(), want_v)
    assert torch.equal(table.cpu(), rows) and n.tolist() == ends
    # into itself, and to a page that is none
    psf.psf_cache_fork(desc, Kp, Vp, table, n, ints([0, 3]), ints([0, 8]), ints([free[8], -1]))
    assert same(Kp.cpu(), want_k) and torch.equal(table[:8].cpu(), rows[:8]) and n[8] == 1 and table[8, 0] == -1


def test_fork_of_a_sequence_with_freed_pages():
    """A parent whose last page has been freed: its child has none there either, and the fresh page stays as it is."""
    desc, Kp, Vp, table, n, free = make_cache([40, 40, 0, 0], 16, 2, 64, "bf16", spare=4)
    table[0, 2], table[1, 1] = -1, -1
    before, rows = Kp.clone(), table.clone()
    psf.psf_cache_fork(desc, Kp, Vp, table, n, ints([0, 1]), ints([2, 3]), ints(free[:2]))
    assert torch.equal(table[2], rows[0]) and n.tolist() == [40] * 4
    assert table[3].tolist() == rows[1, :2].tolist() + [free[1]] + rows[1, 3:].tolist()
    assert same(Kp[free[0]], before[free[0]]) and same(Kp[free[1]], before[int(rows[1, 2])])
    psf.psf_cache_fork(desc, Kp, Vp, table, n, *(torch.empty(0, dtype=torch.int32, device="cuda") for _ in range(3)))


def model_compact(Kp, Vp, table, lengths, page):
    pages, rows = Kp.shape[0], table.tolist()
    used = [row[:max(0, -(-n // page))] for row, n in zip(rows, lengths)]
    marks = {p for row in used for p in row if 0 <= p < pages}
    live = len(marks)
    place = dict(zip(sorted(p for p in marks if p >= live), (p for p in range(live) if p not in marks)))
    for a, b in place.items():
        Kp[b], Vp[b] = Kp[a], Vp[a]
    moved = [[place.get(p, p) if 0 <= p < pages else -1 for p in row] for row in used]
    return torch.tensor([row + [-1] * (table.shape[1] - len(row)) for row in moved], dtype=torch.int32), live


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,page,kv,d,spare", [
    ((1,), 16, 1, 64, 0), ((0, 0), 16, 1, 64, 4), ((100, 33, 0, 7), 16, 2, 64, 40), ((500,) * 9, 8, 1, 8, 33), ((64, 64), 64, 4, 128, 1),
    ((900, 1, 555), 3, 2, 72, 3000), ((2000,) * 3, 1, 1, 8, 70000),
])
def test_compact(lengths, page, kv, d, spare, dtype):
    desc, Kp, Vp, table, n, _ = make_cache(lengths, page, kv, d, dtype, spare=spare, seed=4)
    if len(lengths) > 2:
        table[1, 0] = table[0, 0]                              # a page that two sequences share
        table[0, 2] = -1                                       # a page freed inside a sequence
        table[2, -1] = 0                                       # an entry behind the length
        if lengths[0] > 10 * page:
            table[0, 5] = desc.pages + 3
    want_k, want_v = Kp.cpu(), Vp.cpu()
    want_table, live = model_compact(want_k, want_v, table.cpu(), lengths, page)
    for _ in range(2):                                         # (the same again from the old table)
        new_table, got = psf.psf_cache_compact(desc, Kp, Vp, table, n)
        assert got.item() == live and torch.equal(new_table.cpu(), want_table)
        assert same(Kp.cpu(), want_k) and same(Vp.cpu(), want_v)
    q = torch.randn(len(lengths), kv, 1, d, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).cuda()
    if len(lengths) <= 2:
        assert_within(psf.psf_paged_attn(desc, q, Kp, Vp, new_table, n), *reference(q, Kp, Vp, new_table, lengths, page))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_server_from_prompt_to_forked_continuations(dtype):
    """Normalised rows, prompts through the window attention, their keys and values appended, steps through the paged attention,
    a fork and a compaction between them: every step's row is that of the window attention over the whole sequence."""
    heads, kv, d, page, window, sinks, total = 4, 2, 64, 16, 40, 3, 130
    prompts = [57, 16, 101, 0]
    g = torch.Generator().manual_seed(21)
    td = TYPES[dtype]
    w, b = (1 + 0.1 * torch.randn(d, generator=g)).to(td).cuda(), (0.1 * torch.randn(d, generator=g)).to(td).cuda()
    Q, K = (autograd.layer_norm(torch.randn(4, h, total, d, generator=g).to(td).cuda(), w, b) for h in (heads, kv))
    V = torch.randn(4, kv, total, d, generator=g).to(td).cuda()
    for t in (Q, K, V):
        t[3] = t[0]                                            # the fork continues as its parent does
    whole = psf.psf_window_attn_fwd(psf.make_window_desc(4, heads, total, d, window, sinks, dtype, kv_heads=kv), Q, K, V)
    n = ints(prompts)
    rows = psf.psf_window_attn_fwd(psf.make_window_desc(4, heads, 101, d, window, sinks, dtype, kv_heads=kv),
                                   *(t[:, :, :101].contiguous() for t in (Q, K, V)), lengths=n)
    step = {"bf16": 4 * 2.0 ** -8, "f32": 2.0 ** -17}[dtype]   # two results within r (A + ...) of the same value
    for i, length in enumerate(prompts):
        off = (rows[i, :, :length].double() - whole[i, :, :length].double()).abs()
        assert length == 0 or off.max() <= step * whole.double().abs().max()
    pages = 64
    desc = psf.make_cache_desc(pages, page, kv, d, 4, 9, dtype)
    Kp, Vp = psf.cache_new_pools(desc)
    for pool in (Kp, Vp):
        pool.fill_(float("nan"))
    order = list(range(pages))
    random.Random(5).shuffle(order)
    table = torch.full((4, 9), -1, dtype=torch.int32)
    for i in range(3):
        table[i] = torch.tensor(order[9 * i:9 * i + 9])
    table = table.cuda()
    psf.psf_cache_append(desc, K, V, Kp, Vp, table, ints([0] * 4), counts=n)
    workspace = psf.alloc_paged_workspace(desc, heads)
    for turn in range(20):
        if turn == 5:
            psf.psf_cache_fork(desc, Kp, Vp, table, n, ints([0]), ints([3]), ints([order[40]]))
            table[3, int(n[3]) // page + 1:] = ints(order[41:41 + 8 - int(n[3]) // page])   # pages to come, of its own
        if turn == 11:
            spare = table.clone()
            table, live = psf.psf_cache_compact(desc, Kp, Vp, table, n)
            for pool in (Kp, Vp):
                pool[int(live):] = float("nan")                # free pages may hold anything
            at = int(live)
            for i in range(4):                                 # pages to come, from the free ones
                first = -(-int(n[i]) // page)
                table[i, first:] = ints(list(range(at, at + 9 - first)))
                at += 9 - first
            assert at <= pages and not torch.equal(spare, table)
        active = [i for i in range(4) if i != 3 or turn >= 5]
        at = [min(int(x), total - 1) for x in n]
        take = lambda t: torch.stack([t[i, :, p:p + 1] for i, p in enumerate(at)])
        counts = ints([1 if i in active else 0 for i in range(4)])
        psf.psf_cache_append(desc, take(K), take(V), Kp, Vp, table, n, counts=counts)
        n = n + counts
        o = psf.psf_paged_attn(desc, take(Q), Kp, Vp, table, n, window=window, sinks=sinks, workspace=workspace)
        for i in active:
            want = whole[i, :, at[i]:at[i] + 1].double()
            assert (o[i].double() - want).abs().max() <= step * want.abs().max().clamp(min=1.0), (turn, i)
        if 3 not in active:
            assert not o[3].any()
    assert n.tolist() == [77, 36, 121, 77]


def test_steps_in_a_graph():
    """A step captured once (append, advance, attention) and replayed against the eager calls."""
    desc, Kp, Vp, table, n, _ = make_cache((120, 77), 16, 2, 64, "bf16", seed=11)
    table[1, 5:8] = ints([desc.pages - 1, desc.pages - 2, desc.pages - 3])
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(2, 2, 1, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn(2, 4, 1, 64, generator=g).to(torch.bfloat16).cuda()
    workspace = psf.alloc_paged_workspace(desc, 4)
    live = torch.empty(1, dtype=torch.int32, device="cuda")
    new_table = torch.empty_like(table)

    def step():
        psf.psf_cache_append(desc, k, v, Kp, Vp, table, n)
        n.add_(1)
        psf.psf_cache_compact(desc, Kp2, Vp2, table, n, new_table=new_table, live=live, workspace=room)
        return psf.psf_paged_attn(desc, q, Kp, Vp, table, n, workspace=workspace)

    Kp2, Vp2, room = Kp.clone(), Vp.clone(), psf.alloc_compact_workspace(desc)
    kept = [t.clone() for t in (Kp, Vp, n)]
    eager = [(step().clone(), live.item(), new_table.clone()) for _ in range(4)]
    for t, was in zip((Kp, Vp, n), kept):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o = step()
    for want, pages, places in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and live.item() == pages and torch.equal(new_table, places)
