"""The paged cache against float64 and against the dense calls.

Tolerances of a step, per element, with size = sum_r p_r |v_r| over n rows and e = (D + 8) 2^-24 max_r sum_d |q_d k_rd| / sqrt(D) the
logits' error: weights and sums (2 e + (n + 64) 2^-24), bf16 weights kept to 2^-21 on top; outputs that times size; a cumulative score
that times its increment, and a rounding of 2^-24 of itself."""
import numpy as np
import pytest
import torch

from oracle import uncomp_oracle as O
from tests._util import raw_bits, to_f64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_2410_03090_amd import binding
    c = binding.Context(0, 256 << 20)
    yield c
    c.close()


def _cache(ctx, lens, page, max_pages, D, dtype, seed, spare=3, room=1):
    """Pages handed out in random order, for every head's rows and `room` more; the rest of the pool is NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [min(max_pages, -(-(n + room) // page)) for n in lens]
    order = torch.randperm(sum(need) + spare, generator=g).tolist()
    c = ctx.paged_new(len(lens), len(order), page, max_pages, D, dtype)
    c.K.fill_(float("nan")), c.V.fill_(float("nan")), c.cum.fill_(float("nan"))
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32)
    for h, n in enumerate(need):
        table[h, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    c.table.copy_(table)
    rows = max(max(lens), 1)
    K, V = (torch.randn(len(lens), rows, D, generator=g).to(dtype) for _ in range(2))
    idx = torch.sort(torch.stack([torch.randperm(4 * rows, generator=g)[:rows] for _ in lens]), dim=1)[0].to(torch.int32)
    cum = torch.rand(len(lens), rows, generator=g) * 3
    ctx.paged_append(c, K.to(DEV), V.to(DEV), idx.to(DEV), cum=cum.to(DEV), rows=torch.tensor(lens, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert c.length.cpu().tolist() == list(lens)
    return c, (K, V, idx, cum)


def _rows(c, h, n=None):
    """(K, V, idx, cum) of a head's rows, on the host."""
    page = c.K.shape[1]
    n = int(c.length[h]) if n is None else n
    pages = c.table[h, :-(-n // page)].long()
    return [t[pages].flatten(0, 1)[:n].cpu() for t in (c.K, c.V, c.idx, c.cum)]


def _host(c):
    return [raw_bits(t) for t in (c.K, c.V, c.idx, c.cum, c.table, c.length)]


def _check_step(before, after, q, kn, vn, pos, out, dtype, what):
    """before / after: a head's rows; kn None: nothing joins."""
    K, V, idx, cum = before
    D = q.shape[1]
    if kn is not None:
        K, V = torch.cat([K, kn[None]]), torch.cat([V, vn[None]])
        idx, cum = torch.cat([idx, torch.tensor([pos], dtype=torch.int32)]), torch.cat([cum, torch.zeros(1)])
    assert np.array_equal(raw_bits(K), raw_bits(after[0])) and np.array_equal(raw_bits(V), raw_bits(after[1])), what
    assert torch.equal(idx, after[2]), what
    if len(K) == 0:
        assert (out == 0).all(), what
        return
    k, v, qq = to_f64(K), to_f64(V), to_f64(q)
    z = qq @ k.T / np.sqrt(D)
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    e = (D + 8) * 2.0 ** -24 * (np.abs(qq) @ np.abs(k).T).max(axis=1) / np.sqrt(D)
    rel = 2 * e + (len(k) + 64) * 2.0 ** -24
    size = p @ np.abs(v)
    tol = (rel + (2.0 ** -21 if dtype == torch.bfloat16 else 0.0))[:, None] * size
    err = np.abs(to_f64(out) - p @ v)
    assert (err <= tol).all(), f"{what}: output off by {err.max()}, {(err / tol).max()} of what is allowed"
    want = to_f64(cum) + p.sum(axis=0)
    tol = (rel[:, None] * p).sum(axis=0) + 2.0 ** -24 * (want + 16 * p.sum(axis=0))
    err = np.abs(to_f64(after[3]) - want)
    assert (err <= tol).all(), f"{what}: cum off by {err.max()}, {(err / tol).max()} of what is allowed"


def _token(n, G, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return ((1.5 * torch.randn(n, G, D, generator=g)).to(dtype), torch.randn(n, D, generator=g).to(dtype), torch.randn(n, D, generator=g).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G,D,page", [(1, 128, 16), (4, 128, 64), (7, 128, 32), (16, 128, 256), (4, 64, 16), (8, 64, 128)])
def test_steps_match_float64(ctx, dtype, G, D, page):
    """Lengths around blocks, waves and pages; two tokens in a row; the second finds pages full, which some heads cannot leave."""
    lens = [0, 1, 15, 16, 17, 31, 33, 127, 128, 129, 300, 511, 1000]
    max_pages = -(-1024 // page)
    c, _ = _cache(ctx, lens, page, max_pages, D, dtype, 100 + G, room=1)
    n = len(lens)
    for t in range(2):
        q, kn, vn = _token(n, G, D, dtype, 50 + t)
        pos = torch.full((n,), 5000 + t, dtype=torch.int32)
        before = [_rows(c, h) for h in range(n)]
        fits = [(b[0].shape[0] < max_pages * page) and int(c.table[h, b[0].shape[0] // page]) >= 0 for h, b in enumerate(before)]
        assert t == 1 or all(fits)
        out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos.to(DEV))
        torch.cuda.synchronize()
        for h in range(n):
            _check_step(before[h], _rows(c, h), q[h], kn[h] if fits[h] else None, vn[h], 5000 + t, out[h].cpu(), dtype, f"token {t}, head {h}")


@pytest.mark.parametrize("dtype,lens,page", [(torch.bfloat16, [20011, 7], 128), (torch.bfloat16, [40000], 16), (torch.float32, [9001, 4096], 64)])
def test_long_caches_of_few_heads(ctx, dtype, lens, page):
    G, D = 4, 128
    c, _ = _cache(ctx, lens, page, -(-(max(lens) + 1) // page), D, dtype, 7)
    q, kn, vn = _token(len(lens), G, D, dtype, 8)
    before = [_rows(c, h) for h in range(len(lens))]
    pos = torch.full((len(lens),), 10 ** 6, dtype=torch.int32)
    out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos.to(DEV))
    torch.cuda.synchronize()
    for h in range(len(lens)):
        _check_step(before[h], _rows(c, h), q[h], kn[h], vn[h], 10 ** 6, out[h].cpu(), dtype, f"head {h}")


@pytest.mark.parametrize("heads,lens_to,G", [(1300, 200, 4), (600, 700, 8), (300, 60, 16), (260, 2500, 2), (300, 1500, 16), (30, 1500, 4), (150, 1100, 8), (5, 300, 3)])
def test_many_heads(ctx, heads, lens_to, G):
    """One workgroup a head, or several; every seventh head is checked."""
    dtype, D, page = torch.bfloat16, 128, 32
    g = torch.Generator().manual_seed(heads)
    lens = torch.randint(0, lens_to + 1, (heads,), generator=g).tolist()
    c, _ = _cache(ctx, lens, page, -(-(lens_to + 1) // page), D, dtype, 9)
    q, kn, vn = _token(heads, G, D, dtype, 10)
    pick = list(range(0, heads, 7))
    before = {h: _rows(c, h) for h in pick}
    pos = torch.full((heads,), 10 ** 5, dtype=torch.int32)
    out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos.to(DEV))
    torch.cuda.synchronize()
    assert c.length.cpu().tolist() == [n + 1 for n in lens]
    for h in pick:
        _check_step(before[h], _rows(c, h), q[h], kn[h], vn[h], 10 ** 5, out[h].cpu(), dtype, f"head {h}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_alone_missing_pages_and_lengths_out_of_range(ctx, dtype):
    """No token joins; pages that are none are passed over; lengths are cut to the table."""
    G, D, page = 4, 128, 16
    lens = [100, 100, 40, 0, 64]
    c, _ = _cache(ctx, lens, page, 7, D, dtype, 11)
    whole = [_rows(c, h) for h in range(5)]
    c.table[1, 2], c.table[1, 5], c.table[2, 0] = -1, c.K.shape[0], 2 ** 31 - 1
    c.length[3], c.length[4] = -5, 10 ** 6
    c.table[4, 5:] = -1
    q, kn, vn = _token(5, G, D, dtype, 12)
    out = ctx.paged_step(c, q.to(DEV))
    torch.cuda.synchronize()
    keep = [range(100), [r for r in range(100) if r // 16 not in (2, 5)], range(16, 40), [], None]
    for h in range(4):
        before = [t[list(keep[h])] for t in whole[h]]
        pages = c.table[h].cpu()
        got = [torch.stack([t[int(pages[r // page]), r % page].cpu() for r in keep[h]]) if len(keep[h]) else t.cpu()[0, :0]
               for t in (c.K, c.V, c.idx, c.cum)]
        _check_step(before, got, q[h], None, None, 0, out[h].cpu(), dtype, f"head {h}")
    # the last head's rows end with its pages: rows 64 ... 79 of its fifth page hold NaN, as does its output
    assert out[4].isnan().all()
    # a full table and a missing page: the token is left out, everything else as it was
    c.length[4] = 64
    c.table[0, 6] = -1
    c.length[0] = 96
    before, state = [_rows(c, 0)], _host(c)
    pos = torch.full((5,), 9, dtype=torch.int32, device=DEV)
    c.length[2] = 7 * page
    out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos)
    torch.cuda.synchronize()
    assert c.length.cpu().tolist() == [96, 101, 112, 1, 65]
    _check_step(before[0], _rows(c, 0), q[0], None, None, 9, out[0].cpu(), dtype, "full head")
    assert np.array_equal(state[0][int(c.table[0, 5])], raw_bits(c.K[int(c.table[0, 5])]))


@pytest.mark.parametrize("n,G,D,dtype,max_pages", [(520, 4, 128, torch.bfloat16, 80), (600, 16, 64, torch.float32, 40), (700, 8, 128, torch.bfloat16, 200)])
def test_many_heads_short_and_long(ctx, n, G, D, dtype, max_pages):
    """Short heads, and among them some too long for one workgroup's LDS, at lengths around that (50 KiB of logits), none of them and all of them."""
    page = 64
    short = 50 * 1024 // (G * 4) // 32 * 32
    lens = [(37 * h) % 90 for h in range(n)]
    long = {0: short - 2, 1: short - 1, 2: short, 3: short + 1, 70: min(2 * short, max_pages * page - 3), n // 2: short + 40, n - 1: short + 130}
    for h, m in long.items():
        lens[h] = m
    c, _ = _cache(ctx, lens, page, max_pages, D, dtype, 42, room=3)
    pick = sorted(long) + [4, 5, 69, 71, n - 2]
    for t in range(3):                                                   # (the third without the new token)
        q, kn, vn = _token(n, G, D, dtype, 60 + t)
        before = {h: _rows(c, h) for h in pick}
        pos = torch.full((n,), 10 ** 6 + t, dtype=torch.int32, device=DEV)
        out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos) if t < 2 else ctx.paged_step(c, q.to(DEV))
        torch.cuda.synchronize()
        assert c.length.cpu().tolist() == [m + min(t + 1, 2) for m in lens]
        for h in pick:
            _check_step(before[h], _rows(c, h), q[h], kn[h] if t < 2 else None, vn[h], 10 ** 6 + t, out[h].cpu(), dtype, f"token {t}, head {h}")
    c.length.zero_()
    assert (ctx.paged_step(c, q.to(DEV)) == 0).all() and (c.length == 0).all()
    if G == 16:
        c, _ = _cache(ctx, [short + h % 3 for h in range(n)], page, max_pages, D, dtype, 43)
        before = {h: _rows(c, h) for h in pick}
        out = ctx.paged_step(c, q.to(DEV))
        torch.cuda.synchronize()
        for h in pick:
            _check_step(before[h], _rows(c, h), q[h], None, None, 0, out[h].cpu(), dtype, f"all long, head {h}")


@pytest.mark.parametrize("n,G,max_pages,mib", [(6, 4, 2500, 3), (100, 16, 600, 8), (700, 8, 2500, 24)])
def test_tables_with_more_room_than_the_pool_has_rows(ctx, n, G, max_pages, mib):
    """Tables for thousands of rows a head over a pool of a few pages each: the workspace goes by the pool.  Steps and evictions; a head that counts
    rows without pages leaves the others alone."""
    from paper_2410_03090_amd import binding
    D, page, dtype = 64, 16, torch.bfloat16
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 90, (n,), generator=g).tolist()
    lens[-1] = 300
    c, _ = _cache(ctx, lens, page, max_pages, D, dtype, 40, room=2)
    small = binding.Context(0, mib << 20)
    assert binding.Context.paged_workspace_bytes(n, G, D, max_pages * page) > mib << 20
    pick = [0, 1, 2, n // 2, n - 2, n - 1]
    for t in range(2):
        q, kn, vn = _token(n, G, D, dtype, 80 + t)
        before = {h: _rows(c, h) for h in pick}
        pos = torch.full((n,), 10 ** 6 + t, dtype=torch.int32, device=DEV)
        out = small.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos)
        torch.cuda.synchronize()
        for h in pick:
            _check_step(before[h], _rows(c, h), q[h], kn[h], vn[h], 10 ** 6 + t, out[h].cpu(), dtype, f"token {t}, head {h}")
    _check_evict(small, c, [max(5, m // 2) for m in lens], [10 ** 7] * n, 4)
    c.length[0] = max_pages * page - 1000                                                  # rows that it has no pages for
    before = {h: _rows(c, h) for h in pick[1:]}
    q, kn, vn = _token(n, G, D, dtype, 90)
    out = small.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), torch.full((n,), 2 * 10 ** 6, dtype=torch.int32, device=DEV))
    evicted = small.paged_evict(c, torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV), 10 ** 6)
    torch.cuda.synchronize()
    assert c.length[0] == max_pages * page - 1000 and (evicted == 0).all()
    for h in pick[1:]:
        after = _rows(c, h)
        assert torch.equal(after[2][:-1], before[h][2]) and out[h].isfinite().all()
    small.close()


def test_infinite_values_and_logits(ctx):
    G, D, page = 2, 128, 32
    c, _ = _cache(ctx, [200, 200, 200], page, 7, D, torch.bfloat16, 13)
    q, kn, vn = _token(3, G, D, torch.bfloat16, 14)
    q = q.abs()
    at = [(int(c.table[h, 3]), 5) for h in range(3)]
    c.V[at[0]][9], c.V[at[0]][10] = float("inf"), float("-inf")
    c.K[at[1]][0] = float("-inf")                                # no weight
    c.K[at[2]][0] = float("inf")                                 # no normaliser
    before = _rows(c, 1)
    out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), torch.full((3,), 900, dtype=torch.int32, device=DEV)).cpu()
    torch.cuda.synchronize()
    assert (out[0, :, 9] == float("inf")).all() and (out[0, :, 10] == float("-inf")).all()
    rest = [d for d in range(D) if d not in (9, 10)]
    assert out[0][:, rest].isfinite().all()
    keep = [r for r in range(201) if r != 101]
    after = _rows(c, 1)
    assert after[3][101] == before[3][101]
    _check_step([t[[r for r in range(200) if r != 101]] for t in before], [t[keep] for t in after], q[1], kn[1], vn[1], 900, out[1], torch.bfloat16, "-inf")
    assert out[2].isnan().all()


def test_equals_the_dense_step(ctx):
    """Without evictions the dense and the paged step are the same operator."""
    n, G, D, cap, w = 24, 4, 128, 640, 32
    g = torch.Generator().manual_seed(15)
    lens = torch.randint(1, cap - 8, (n,), generator=g).tolist()
    c, (K, V, idx, cum) = _cache(ctx, lens, 64, cap // 64, D, torch.bfloat16, 16, room=8)
    pad = lambda t: torch.nn.functional.pad(t, (0, 0, 0, cap - t.shape[1]) if t.dim() == 3 else (0, cap - t.shape[1])).contiguous().to(DEV)  # noqa: E731
    Kc, Vc, ic, cc = pad(K), pad(V), pad(idx), pad(cum)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    big = torch.full((n,), cap, dtype=torch.int32, device=DEV)
    for t in range(5):
        q, kn, vn = (x.to(DEV) for x in _token(n, G, D, torch.bfloat16, 60 + t))
        pos = torch.full((n,), 10000 + t, dtype=torch.int32, device=DEV)
        dense, _ = ctx.decode_step(q, kn, vn, pos, big, w, Kc, Vc, ic, cc, ln)
        paged = ctx.paged_step(c, q, kn, vn, pos)
        torch.cuda.synchronize()
        assert torch.equal(ln, c.length)
        np.testing.assert_allclose(paged.cpu().numpy(), dense.cpu().numpy(), rtol=0, atol=4e-5 * float(V.float().abs().max()))
        for h in range(n):
            np.testing.assert_allclose(_rows(c, h)[3].numpy(), cc[h, :int(ln[h])].cpu().numpy(), rtol=4e-5, atol=4e-6)


@pytest.mark.parametrize("dtype,D,page", [(torch.bfloat16, 128, 64), (torch.float32, 64, 16), (torch.bfloat16, 64, 32), (torch.float32, 128, 256)])
def test_append_takes_what_fits(ctx, dtype, D, page):
    n, cap = 6, 70
    g = torch.Generator().manual_seed(17)
    c = ctx.paged_new(n, 40, page, 5, D, dtype)
    table = torch.randperm(40, generator=g)[: n * 5].view(n, 5).to(torch.int32)
    table[2, 1], table[3, 0] = -1, 40
    c.table.copy_(table)
    # every second row of a wider tensor, heads in the middle
    K = torch.randn(cap, n, 2 * D, generator=g).to(dtype)[..., :D].transpose(0, 1)
    V = torch.randn(cap, n, 2 * D, generator=g).to(dtype)[..., :D].transpose(0, 1)
    idx = torch.randint(0, 10 ** 6, (n, cap), generator=g, dtype=torch.int32)
    cum = torch.rand(n, cap, generator=g)
    dev = lambda t: torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=DEV).copy_(t)  # noqa: E731
    offered = [70, 0, 70, 9, 300, -4]
    want = [[] for _ in range(n)]
    for call in range(6):
        ctx.paged_append(c, dev(K), dev(V), idx.to(DEV), cum=cum.to(DEV) if call % 2 == 0 else None,
                         rows=torch.tensor(offered, dtype=torch.int32, device=DEV) if call < 5 else None)
        torch.cuda.synchronize()
        for h in range(n):
            m = cap if call == 5 else min(max(offered[h], 0), cap)
            room = {2: page, 3: 0}.get(h, 5 * page) - len(want[h])
            want[h] += [(r, call % 2 == 0) for r in range(min(m, room))]
        assert c.length.cpu().tolist() == [len(x) for x in want]
    for h in range(n):
        if not want[h]:
            continue
        k, v, i, s = _rows(c, h)
        r = [x for x, _ in want[h]]
        assert np.array_equal(raw_bits(k), raw_bits(K[h][r])) and np.array_equal(raw_bits(v), raw_bits(V[h][r]))
        assert torch.equal(i, idx[h][r])
        assert torch.equal(s, torch.where(torch.tensor([b for _, b in want[h]]), cum[h][r], 0.0))
    free = sorted(set(range(40)) - set(table.flatten().tolist()))
    assert (c.K[free] == 0).all() and (c.idx[free] == -1).all()


def _check_evict(ctx, c, budget, pos, w):
    n = c.length.numel()
    before = [_rows(c, h) for h in range(n)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    evicted = ctx.paged_evict(c, i32(budget), i32(pos), w)
    torch.cuda.synchronize()
    for h in range(n):
        order = O.evict_lowest(before[h][3].numpy(), before[h][2].numpy(), budget[h], pos[h], w)
        assert int(c.length[h]) == len(order) and int(evicted[h]) == len(before[h][3]) - len(order), h
        for a, b in zip(_rows(c, h), before[h]):
            assert np.array_equal(raw_bits(a), raw_bits(b[order])), h


@pytest.mark.parametrize("max_pages", [64, 1100])
def test_evict_short_and_long_heads_together(ctx, max_pages):
    """More heads than get a workgroup each, lengths around what a wave keeps in its registers; tables with room for 4096 rows and for 70400."""
    n, page = 520, 64
    lens = [(53 * h) % 120 for h in range(n)]
    for i, m in enumerate((2046, 2047, 2048, 2049, 2050, 3000, 4000)):
        lens[71 * i] = m
    c, _ = _cache(ctx, lens, page, max_pages, 64, torch.bfloat16, 44)
    budget = [m // 2 + h % 3 for h, m in enumerate(lens)]
    pos = [4 * max(lens) if h % 5 else 200 for h in range(n)]            # (few rows old enough in some)
    _check_evict(ctx, c, budget, pos, 4)
    _check_evict(ctx, c, [b // 2 for b in budget], pos, 2)


@pytest.mark.parametrize("lens", [[1016, 200, 65, 700], [1016, 200, 1400, 1500], [2600, 700, 129, 2000]])
def test_evict_of_rows_that_are_all_alike(ctx, lens):
    """One score and one position for hundreds of rows, more than a lane's or a thread's: the first rows leave, down to the budget exactly."""
    page = 32
    c, _ = _cache(ctx, lens, page, -(-(max(lens) + 1) // page), 64, torch.bfloat16, 41)
    c.cum.fill_(0.5), c.idx.fill_(77)
    _check_evict(ctx, c, [n // 2 for n in lens], [100] * 4, 4)
    _check_evict(ctx, c, [n // 2 - 1 for n in lens], [100] * 4, 4)
    for h, n in enumerate(lens):                                         # a third of the rows at one position more, some of more weight
        rows = torch.arange(n // 2 - 1, device=DEV)
        at = c.table[h, rows // page].long(), rows % page
        c.idx[at] = torch.where(rows % 3 == 0, 78, 77).int()
        c.cum[at] = torch.where(rows % 7 == 0, 0.75, 0.5)
    _check_evict(ctx, c, [n // 4 for n in lens], [100] * 4, 4)


@pytest.mark.parametrize("dtype,D,page", [(torch.bfloat16, 128, 64), (torch.float32, 128, 16), (torch.bfloat16, 64, 32), (torch.float32, 64, 256)])
def test_evict_keeps_the_rows_of_most_weight(ctx, dtype, D, page):
    lens = [0, 1, 5, 64, 100, 300, 1000, 1023, 1024, 1500, 700]
    c, _ = _cache(ctx, lens, page, -(-1600 // page), D, dtype, 18)
    budget = [4, 0, 5, 10, 99, 20, 500, 1022, 0, 1499, -7]
    pos = [4 * n for n in lens]
    _check_evict(ctx, c, budget, pos, 8)
    _check_evict(ctx, c, [b // 2 for b in budget], pos, 3)


def test_evict_ties_infinities_and_nothing_old_enough(ctx):
    """Equal scores go by position, equal positions by row; NaN last; rows that are too recent stay although the head is above its budget."""
    lens = [400, 400, 400, 400, 400, 2600]
    c, _ = _cache(ctx, lens, 32, 82, 128, torch.bfloat16, 19)
    g = torch.Generator().manual_seed(20)
    page = 32

    def put(t, h, values):
        for r in range(0, len(values), page):
            t[int(c.table[h, r // page]), :len(values[r:r + page])] = values[r:r + page].to(DEV)

    put(c.cum, 0, torch.randint(0, 3, (400,), generator=g).float())
    put(c.cum, 1, torch.zeros(400))
    put(c.idx, 1, torch.randint(0, 5, (400,), generator=g, dtype=torch.int32))
    odd = torch.tensor([float("nan"), float("inf"), float("-inf"), 0.0, -0.0, 1e-45, -1.0])
    put(c.cum, 2, odd[torch.randint(0, 7, (400,), generator=g)])
    put(c.cum, 5, torch.randint(0, 2, (2600,), generator=g).float())
    put(c.idx, 5, torch.randperm(2600, generator=g).to(torch.int32))
    _check_evict(ctx, c, [200, 123, 90, 10, 10, 1111], [2000, 2000, 2000, 300, -(2 ** 31), 2 ** 31 - 1], 16)
    _check_evict(ctx, c, [100, 23, 30, 10, 10, 1110], [2000, 2000, 2000, 300, 2 ** 31 - 1, 2000], 0)


@pytest.mark.parametrize("max_pages", [20, 60, 1200])
def test_evict_leaves_a_head_that_lacks_a_page(ctx, max_pages):
    """Tables of up to 1024 rows, up to 2048 and beyond."""
    lens = [1000, 1000, 1000]
    c, _ = _cache(ctx, lens, 32 if max_pages > 20 else 64, max_pages, 64, torch.bfloat16, 26)
    c.table[1, 3] = -1
    c.length[2] = 10 ** 6                                                # cut to the table's rows, whose later pages are none
    before = _host(c)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kept = _rows(c, 0)
    evicted = ctx.paged_evict(c, i32([100] * 3), i32([10 ** 6] * 3), 4)
    torch.cuda.synchronize()
    assert evicted.cpu().tolist() == [900, 0, 0] and c.length.cpu().tolist() == [100, 1000, 10 ** 6]
    order = O.evict_lowest(kept[3].numpy(), kept[2].numpy(), 100, 10 ** 6, 4)
    assert np.array_equal(raw_bits(_rows(c, 0)[0]), raw_bits(kept[0][order]))
    mine = c.table[0, : -(-1000 // c.K.shape[1])].cpu().tolist()
    others = [p for p in range(c.K.shape[0]) if p not in mine]
    for a, b in zip(_host(c)[:4], before[:4]):
        assert np.array_equal(a[others], b[others])


def test_evict_keys_over_the_whole_range_of_floats(ctx):
    """The widest range of keys a search can meet, in tables of every size: negative, tiny, huge, infinite and NaN scores."""
    g = torch.Generator().manual_seed(27)
    for lens, max_pages in (([900, 31], 32), ([1900, 2000], 64), ([5000, 2500], 200), ([70000], 2200)):
        c, _ = _cache(ctx, lens, 32, max_pages, 64, torch.bfloat16, 28)
        bits = torch.randint(-(2 ** 31), 2 ** 31 - 1, c.cum.shape, generator=g, dtype=torch.int64).to(torch.int32)
        c.cum.copy_(bits.view(torch.float32))
        _check_evict(ctx, c, [n // 2 for n in lens], [10 ** 6] * len(lens), 5)
        _check_evict(ctx, c, [n // 2 - 1 for n in lens], [10 ** 6] * len(lens), 5)


@pytest.mark.parametrize("heads,rows", [(2, 50000), (40, 9000), (900, 500)])
def test_evict_at_length(ctx, heads, rows):
    lens = [rows - (h * 37) % (rows // 2) for h in range(heads)]
    c, _ = _cache(ctx, lens, 128, -(-rows // 128) + 1, 64, torch.bfloat16, 21)
    pick = list(range(0, heads, max(1, heads // 5)))
    before = {h: _rows(c, h) for h in pick}
    budget = [n // 3 + h for h, n in enumerate(lens)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ctx.paged_evict(c, i32(budget), i32([4 * rows] * heads), 64)
    torch.cuda.synchronize()
    assert c.length.cpu().tolist() == [min(n, b) for n, b in zip(lens, budget)]     # some budgets lie above the rows
    for h in pick:
        order = O.evict_lowest(before[h][3].numpy(), before[h][2].numpy(), budget[h], 4 * rows, 64)
        for a, b in zip(_rows(c, h), before[h]):
            assert np.array_equal(raw_bits(a), raw_bits(b[order])), h


def test_prompt_to_pages_to_tokens_to_eviction(ctx):
    """The calls in the order of their use: attention over the prompt, its normalisers into the score, selection, cumulative scores,
    pages, tokens, eviction; every stage against float64 on the stage's own inputs."""
    B, H, G, N, w, D, cap, page = 1, 4, 4, 600, 16, 128, 160, 32
    g = torch.Generator().manual_seed(22)
    K, V = (torch.randn(B, H, N, D, generator=g).to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(B, H * G, N, D, generator=g).to(torch.bfloat16)
    Kd, Vd, Qd = K.to(DEV), V.to(DEV), Q.to(DEV)
    budget = torch.tensor([[160, 128, 96, 33]], dtype=torch.int32, device=DEV)
    _, lse = ctx.prefill_attention(Qd, Kd, Vd, G)
    score = ctx.window_score(Qd[:, :, N - w:].contiguous(), Kd, G, lse=lse[:, :, N - w:].contiguous())
    Kc, Vc, idx, ln = ctx.select_gather(score, budget, Kd, Vd, w, cap)
    cum = ctx.decode_init(score, idx, ln, N, w)
    n = B * H
    c = ctx.paged_new(n, 40, page, 8, D)
    c.table.copy_(torch.randperm(40, generator=g)[: n * 8].view(n, 8).to(torch.int32))
    ctx.paged_append(c, Kc.view(n, cap, D), Vc.view(n, cap, D), idx.view(n, cap), cum=cum.view(n, cap), rows=ln.view(n))
    torch.cuda.synchronize()
    sref = O.window_score(to_f64(Q[:, :, N - w:]), to_f64(K), G, 7)
    np.testing.assert_allclose(score.cpu().numpy(), sref, rtol=4e-5)
    for h in range(n):
        k, v, i, s = _rows(c, h)
        assert np.array_equal(raw_bits(k), raw_bits(K[0, h][i.long()])) and np.array_equal(raw_bits(v), raw_bits(V[0, h][i.long()]))
    for t in range(40):
        q, kn, vn = _token(n, G, D, torch.bfloat16, 70 + t)
        before = [_rows(c, h) for h in range(n)]
        pos = torch.full((n,), N + t, dtype=torch.int32, device=DEV)
        out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), pos)
        torch.cuda.synchronize()
        for h in range(n):
            _check_step(before[h], _rows(c, h), q[h], kn[h], vn[h], N + t, out[h].cpu(), torch.bfloat16, f"token {t}, head {h}")
        if t % 16 == 15:
            _check_evict(ctx, c, budget.view(-1).cpu().tolist(), [N + t] * n, w)
            assert c.length.cpu().tolist() == budget.view(-1).cpu().tolist()


def test_graphs_and_streams(ctx):
    """A step and an eviction captured; replays on new contents, eager work between them; another stream."""
    lens, page, D, G, w = [500, 70, 333], 32, 128, 4, 8
    c, _ = _cache(ctx, lens, page, 20, D, torch.bfloat16, 23, room=40)
    q, kn, vn = (x.to(DEV) for x in _token(3, G, D, torch.bfloat16, 24))
    pos = torch.full((3,), 5000, dtype=torch.int32, device=DEV)
    budget = torch.tensor([400, 60, 300], dtype=torch.int32, device=DEV)
    out, evicted = torch.zeros(3, G, D, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)

    def call():
        ctx.paged_step(c, q, kn, vn, pos, out=out)
        ctx.paged_evict(c, budget, pos, w, evicted=evicted)

    keep = [t.clone() for t in c]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    first = [t.clone() for t in c] + [out.clone(), evicted.clone()]
    for a, b in zip(c, keep):
        a.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in range(3):
        for a, b in zip(c, keep):
            a.copy_(b)
        q.copy_(_token(3, G, D, torch.bfloat16, 24 + t)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in c] + [out.clone(), evicted.clone()]
        for a, b in zip(c, keep):
            a.copy_(b)
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, list(c) + [out, evicted]):
            assert torch.equal(a.nan_to_num(77.0), b.nan_to_num(77.0))
        if t == 0:
            for a, b in zip(got, first):
                assert torch.equal(a.nan_to_num(77.0), b.nan_to_num(77.0))


def test_refusals(ctx):
    from paper_2410_03090_amd import binding
    lib = binding.load_library()
    c, _ = _cache(ctx, [20, 30], 16, 4, 128, torch.bfloat16, 25)
    state = _host(c)
    t = torch.zeros(1 << 16, dtype=torch.bfloat16, device=DEV)
    p, h = t.data_ptr(), ctx.handle
    c2 = binding.ctypes.c_int64 * 2

    def cache(**kw):
        s = binding._PagedCacheStruct(c.K.data_ptr(), c.V.data_ptr(), c.idx.data_ptr(), c.cum.data_ptr(), c.table.data_ptr(),
                                      c.length.data_ptr(), binding.BF16, 2, c.K.shape[0], 16, 4, 128)
        for k, v in kw.items():
            setattr(s, k, v)
        return binding.ctypes.byref(s)

    calls = [lambda s: lib.uncomp_paged_append(h, s, p, p, p, None, None, 8, c2(1024, 128), None),
             lambda s: lib.uncomp_paged_step(h, s, p, 4, p, p, p, p, None),
             lambda s: lib.uncomp_paged_evict(h, s, p, p, 4, None, None)]
    for f in calls:
        assert f(None) == binding.ERR_INVALID_ARG
        for kw in (dict(K_pages=None), dict(V_pages=None), dict(idx_pages=None), dict(cum_pages=None), dict(table=None), dict(len=None),
                   dict(n_heads=0), dict(n_pages=0), dict(max_pages=-1), dict(K_pages=c.K.data_ptr() + 8), dict(len=c.length.data_ptr() + 1)):
            assert f(cache(**kw)) == binding.ERR_INVALID_ARG, kw
        for kw in (dict(dtype=2), dict(D=96), dict(page=48), dict(page=8), dict(page=512), dict(max_pages=1 << 23), dict(n_heads=1 << 22)):
            assert f(cache(**kw)) == binding.ERR_UNSUPPORTED, kw
        assert b"paged" in lib.uncomp_last_error(h)
    ok = cache()
    append = lambda **kw: lib.uncomp_paged_append(*{**dict(c=h, s=ok, K=p, V=p, idx=p, cum=None, n=None, rows=8, st=c2(1024, 128), stream=None), **kw}.values())  # noqa: E731
    for kw in (dict(c=None), dict(K=None), dict(V=None), dict(idx=None), dict(st=None), dict(rows=0), dict(st=c2(1024, 120)), dict(st=c2(-8, 128)),
               dict(st=c2(1028, 128)), dict(K=p + 8), dict(idx=p + 2)):
        assert append(**kw) == binding.ERR_INVALID_ARG, kw
    step = lambda **kw: lib.uncomp_paged_step(*{**dict(c=h, s=ok, q=p, G=4, k=p, v=p, pos=p, out=p, stream=None), **kw}.values())  # noqa: E731
    for kw in (dict(c=None), dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(q=p + 8), dict(out=p + 2)):
        assert step(**kw) == binding.ERR_INVALID_ARG, kw
    for kw in (dict(G=0), dict(G=17)):
        assert step(**kw) == binding.ERR_UNSUPPORTED, kw
    evict = lambda **kw: lib.uncomp_paged_evict(*{**dict(c=h, s=ok, b=p, pos=p, w=4, ev=None, stream=None), **kw}.values())  # noqa: E731
    for kw in (dict(c=None), dict(b=None), dict(pos=None), dict(w=-1), dict(b=p + 2)):
        assert evict(**kw) == binding.ERR_INVALID_ARG, kw
    small = binding.Context(0, 1 << 15)
    big = cache(max_pages=1 << 16, n_pages=1 << 20)
    assert lib.uncomp_paged_step(small.handle, big, p, 4, p, p, p, p, None) == binding.ERR_WORKSPACE
    assert lib.uncomp_paged_evict(small.handle, big, p, p, 4, None, None) == binding.ERR_WORKSPACE
    assert b"workspace" in lib.uncomp_last_error(small.handle)
    torch.cuda.synchronize()
    small.close()
    for a, b in zip(state, _host(c)):
        assert np.array_equal(a, b)


def test_append_strides_of_one_head_or_one_row(ctx):
    """A dimension of one entry has any stride: K and V need not agree there."""
    D, cap = 128, 40
    g = torch.Generator().manual_seed(52)
    wide = torch.randn(cap, 3 * D, generator=g).to(torch.bfloat16).to(DEV)
    K = wide[:, :D].unsqueeze(0)
    V = wide.view(cap, 3, D)[:, 1:2].transpose(0, 1)
    assert K.stride(0) != V.stride(0) and K.stride(1) == V.stride(1)
    idx = torch.arange(cap, dtype=torch.int32, device=DEV)[None]
    c = ctx.paged_new(1, 4, 16, 4, D)
    c.table.copy_(torch.tensor([[2, 0, 3, 1]], dtype=torch.int32))
    ctx.paged_append(c, K, V, idx)
    torch.cuda.synchronize()
    k, v, i, s = _rows(c, 0)
    assert len(k) == cap and torch.equal(k, K[0].cpu()) and torch.equal(v, V[0].cpu()) and torch.equal(i, idx[0].cpu()) and (s == 0).all()
    n = 5
    K = torch.randn(n, 2, D, generator=g).to(torch.bfloat16).to(DEV)[:, :1]
    V = torch.randn(n, 2 * D, generator=g).to(torch.bfloat16).to(DEV)[:, :D].as_strided((n, 1, D), (2 * D, 8, 1))
    c = ctx.paged_new(n, n, 16, 1, D)
    c.table.copy_(torch.arange(n, dtype=torch.int32).view(n, 1))
    ctx.paged_append(c, K, V, torch.full((n, 1), 3, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for h in range(n):
        k, v, i, _ = _rows(c, h)
        assert torch.equal(k, K[h].cpu()) and torch.equal(v, V[h].cpu()) and i.tolist() == [3]


@pytest.mark.parametrize("n,lens_to,long,max_pages,G,dtype", [(40, 60, 0, 2, 4, torch.bfloat16), (2, 5, 20011, 314, 4, torch.bfloat16),
                                                              (3, 9, 9001, 600, 7, torch.float32), (600, 60, 4000, 90, 8, torch.bfloat16),
                                                              (700, 20, 2000, 700, 16, torch.float32)])
def test_steps_without_outputs(ctx, n, lens_to, long, max_pages, G, dtype):
    """One workgroup a head, heads in parts, listed heads, workspace by the tables and by the pool: without outputs the cache becomes what it becomes
    with them."""
    D, page = 64, 64
    lens = [(37 * h) % (lens_to + 1) for h in range(n)]
    if long:
        lens[0], lens[n // 2] = long, long - 77
    pair = [_cache(ctx, lens, page, max_pages, D, dtype, 51, room=2)[0] for _ in range(2)]
    pick = sorted({0, 1, n // 2, n - 1})
    for t in range(2):
        q, kn, vn = _token(n, G, D, dtype, 95 + t)
        before = {h: _rows(pair[0], h) for h in pick}
        args = [x.to(DEV) for x in (q, kn, vn)] + [torch.full((n,), 10 ** 6 + t, dtype=torch.int32, device=DEV)]
        out = ctx.paged_step(pair[0], *args)
        assert ctx.paged_step(pair[1], *args, want_out=False) is None
        torch.cuda.synchronize()
        for a, b in zip(_host(pair[0]), _host(pair[1])):
            assert np.array_equal(a, b)
        for h in pick:
            _check_step(before[h], _rows(pair[1], h), q[h], kn[h], vn[h], 10 ** 6 + t, out[h].cpu(), dtype, f"token {t}, head {h}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_smallest_cache(ctx, dtype):
    """One head with one page of sixteen rows: empty, growing row by row until it is full, cut to one row, cut to none."""
    G, D = 1, 64
    c = ctx.paged_new(1, 1, 16, 1, D, dtype)
    c.table.zero_()
    for t in range(18):
        q, kn, vn = _token(1, G, D, dtype, 200 + t)
        before = _rows(c, 0)
        out = ctx.paged_step(c, q.to(DEV), kn.to(DEV), vn.to(DEV), torch.full((1,), t, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        assert int(c.length[0]) == min(t + 1, 16)
        _check_step(before, _rows(c, 0), q[0], kn[0] if t < 16 else None, vn[0], t, out[0].cpu(), dtype, f"token {t}")
    _check_evict(ctx, c, [1], [17], 0)
    assert int(c.length[0]) == 1
    _check_evict(ctx, c, [0], [17], 0)
    assert int(c.length[0]) == 0
    assert (ctx.paged_step(c, q.to(DEV)) == 0).all() and int(c.length[0]) == 0
