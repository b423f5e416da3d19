"""Speed and accuracy cases of prompt attention and of the paged cache, in plain torch operations or through the library.

Four operators that a program serving a compressed cache calls one after the other:

  attention  causal attention over whole prompts (grouped heads, packed sequences, earlier keys) with its row normalisers
  append     the compacted cache of a prompt joins pages, every head with a length and a page table of its own
  step       one generated token: it joins every head's pages, its queries attend, the rows' attention weights accumulate
  evict      heads above their budget give up the rows of least accumulated weight and close the gaps

Head counts, prompt lengths and budgets are those of the benchmark configurations, with odd and ragged ones between them; keys
are low rank plus noise, as the benchmark's.
"""
import math

import torch

own = False

DEV = "cuda:0"
ROOM = 64                 # generated tokens that fit behind a head's rows before an eviction is due
RING = 16                 # generated tokens kept at hand by a step case


def _attn(name, dtype, H, G, D, seqs):
    """seqs: "n" or "n+m" for every sequence, n queries after m earlier keys."""
    return dict(name=name, kind="attention", dtype=dtype, H=H, G=G, D=D, seqs=seqs)


def _paged(name, kind, dtype, heads, G, D, rows, page, **kw):
    """rows: the longest head's; the eight head groups hold 12 / 12, 11 / 12, ... 5 / 12 of it."""
    return dict(name=name, kind=kind, dtype=dtype, heads=heads, G=G, D=D, rows=rows, page=page, **kw)


def listed():
    return [
        # a short fp32 prompt, one layer: the smallest attention call
        _attn("attn_fp32_1k", "f32", 8, 4, 128, "1024"),
        # one layer of an ordinary 8K prompt
        _attn("attn_8k", "bf16", 8, 4, 128, "8192"),
        # one layer of a batch of ragged prompts with 64-wide heads, some of which continue an earlier part
        _attn("attn_packed_d64", "bf16", 8, 4, 64, "5003,17,1+3000,2048,333+4091,64,129,1021+511,8,3500"),
        # one layer of a 32K prompt: the largest
        _attn("attn_32k", "bf16", 8, 4, 128, "32768"),
        # the compacted cache of all layers of one prompt moves into pages
        _paged("append_8b_all", "append", "bf16", 256, 4, 128, 2736, 64),
        # one layer's cache of 64-wide fp32 heads, pages of 16 rows, an odd number of rows
        _paged("append_f32_d64", "append", "f32", 8, 4, 64, 517, 16),
        # one token of one sequence, one layer: the smallest step, latency counts
        _paged("step_8b_layer", "step", "bf16", 8, 4, 128, 2736, 64),
        # one token of one sequence, the heads of all layers in one call
        _paged("step_8b_all", "step", "bf16", 256, 4, 128, 2736, 64),
        # one token of eight sequences of the 80-layer model
        _paged("step_70b_b8", "step", "bf16", 5120, 8, 128, 1016, 32),
        # one token of one sequence over one layer's whole 128K cache
        _paged("step_128k", "step", "bf16", 8, 4, 128, 131072, 128),
        # 64 generated tokens behind the budgets of eight sequences of the 80-layer model
        _paged("evict_70b_b8", "evict", "bf16", 5120, 8, 128, 1016, 32, keep=0.94),
        # memory is short: every head of one sequence is cut to a quarter
        _paged("evict_cut", "evict", "bf16", 256, 4, 128, 8192, 64, keep=0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["attention", "append", "step", "evict"], [5, 2, 5, 2])[0]
    dtype = rng.choices(["bf16", "f32"], [4, 1])[0]
    D = rng.choices([128, 64], [3, 1])[0]
    if kind == "attention":
        H, G, n = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 7, 8]), rng.choice([1, 1, 1, 2, 5, 12])
        seqs = []
        room = 32 * 32768.0 ** 2 / 2 / (16 if dtype == "f32" else 1)             # visible pairs of the largest case
        for _ in range(n):
            q = _log_int(rng, 1, 32768)
            earlier = _log_int(rng, 1, 32768) if rng.random() < 0.3 else 0
            while H * G * q * (earlier + q / 2.0) > room / n:
                q, earlier = q * 3 // 4 + (q < 4), earlier * 3 // 4
                if q <= 1:
                    break
            seqs.append("%d+%d" % (q, earlier) if earlier else "%d" % q)
        return dict(kind=kind, dtype=dtype, H=H, G=G, D=D, seqs=",".join(seqs))
    case = dict(kind=kind, dtype=dtype, heads=_log_int(rng, 1, 5120), G=rng.choice([1, 2, 4, 4, 7, 8, 16]), D=D,
                rows=_log_int(rng, 2, 131072), page=rng.choice([16, 32, 64, 64, 128, 256]))
    if kind == "evict":
        case["keep"] = rng.choice([0.94, 0.75, 0.5, 0.25])
    limit = 5120 * 1016 * 128 * 2 // (4 if kind == "append" else 1)
    while case["heads"] * (case["rows"] + ROOM) * D * _elem(case) > limit:
        big = "heads" if case["heads"] * 32 > case["rows"] else "rows"
        case[big] = case[big] * 3 // 4 + 1
    return case


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _bits(t):
    """Copies of rows are compared as whole numbers."""
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def _factors(g, n, R, D):
    """[n, R, D] right factors of n heads, each of a rank of its own: U @ factor has variance 1 / rank."""
    ranks = torch.randint(4, R + 1, (n, 1, 1), generator=g, device=DEV)
    return torch.where(torch.arange(R, device=DEV)[None, :, None] < ranks, torch.randn(n, R, D, generator=g, device=DEV), 0.0) / ranks


# ---- attention over whole prompts -----------------------------------------------------------------------------------


def _seqs(case):
    """[(queries, keys)] of every sequence."""
    pairs = [tuple(int(x) for x in s.split("+")) for s in case["seqs"].split(",")]
    return [(p[0], sum(p)) for p in pairs]


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def _prepare_attention(case, seed):
    """Projections as a model leaves them, token by token: Q [T, H*G, D], K and V [T, H, D], seen head first."""
    H, G, D, dt = case["H"], case["G"], case["D"], _dtype(case)
    seqs = _seqs(case)
    qs, ks = _starts([a for a, _ in seqs]), _starts([b for _, b in seqs])
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *sh: torch.randn(*sh, generator=g, device=DEV)  # noqa: E731
    f = _factors(g, H, 96, D)
    Q = torch.empty(qs[-1], H, G, D, dtype=dt, device=DEV)
    K = torch.empty(ks[-1], H, D, dtype=dt, device=DEV)
    for h in range(H):
        K[:, h] = rand(ks[-1], 96) @ f[h] + 0.1 * rand(ks[-1], D)
        for a in range(G):
            Q[:, h, a] = 1.5 * (rand(qs[-1], 96) @ f[h] + 0.1 * rand(qs[-1], D))
    V = rand(ks[-1], H, D).to(dt)
    state = dict(case=case, seqs=seqs, qs=qs, ks=ks, Q=Q.view(qs[-1], H * G, D).transpose(0, 1), K=K.transpose(0, 1), V=V.transpose(0, 1))
    state["q_first"] = torch.tensor(qs, dtype=torch.int32, device=DEV)
    state["k_first"] = torch.tensor(ks, dtype=torch.int32, device=DEV)
    state["out"] = torch.empty(qs[-1], H * G, D, dtype=dt, device=DEV).transpose(0, 1)
    state["lse"] = torch.empty(H * G, qs[-1], dtype=torch.float32, device=DEV)
    if own:
        from paper_2410_03090_amd import binding
        state["ctx"] = binding.Context(0, binding.Context.prefill_attention_workspace_bytes(len(seqs), H, G, D, qs[-1], ks[-1]))
    return state


def _attention_plain(s):
    """Blocks of queries, each over the keys that its last row sees."""
    G, D = s["case"]["G"], s["case"]["D"]
    for (nq, nk), q0, k0 in zip(s["seqs"], s["qs"], s["ks"]):
        step = max(1, min(nq, (1 << 26) // (G * nk)))
        for h in range(s["case"]["H"]):
            heads = slice(h * G, (h + 1) * G)
            k, v = s["K"][h, k0:k0 + nk].float(), s["V"][h, k0:k0 + nk].float()
            for a in range(0, nq, step):
                b = min(nq, a + step)
                seen = nk - nq + b
                rows = slice(q0 + a, q0 + b)
                logits = (s["Q"][heads, rows].float().reshape(-1, D) @ k[:seen].T).view(G, b - a, seen) / math.sqrt(D)
                late = torch.arange(seen, device=DEV)[None, :] > (nk - nq + torch.arange(a, b, device=DEV))[:, None]
                logits.masked_fill_(late, float("-inf"))
                top = logits.amax(dim=2, keepdim=True)
                p = (logits - top).exp_()
                total = p.sum(dim=2, keepdim=True)
                s["out"][heads, rows] = ((p.view(-1, seen) @ v[:seen]).view(G, b - a, D) / total).to(s["out"].dtype)
                s["lse"][heads, rows] = (top + total.log())[..., 0]
    return s["out"], s["lse"]


def _run_attention(s):
    if own:
        return s["ctx"].prefill_attention(s["Q"], s["K"], s["V"], s["case"]["G"], q_first=s["q_first"], k_first=s["k_first"],
                                          out=s["out"], lse=s["lse"])
    return _attention_plain(s)


def _exact_attention(case, seed):
    s = _prepare_attention(case, seed)
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for i, (nq, nk) in enumerate(s["seqs"]):
        key = torch.arange(nk, device=DEV)
        for head in range(case["H"] * case["G"]):
            k = s["K"][head // case["G"], s["ks"][i]:s["ks"][i + 1]].double()
            v = s["V"][head // case["G"], s["ks"][i]:s["ks"][i + 1]].double()
            for part in torch.arange(nq, device=DEV).split(2048):
                q = s["Q"][head, s["qs"][i] + part].double() * case["D"] ** -0.5
                last = nk - nq + part
                n = int(last[-1]) + 1
                z = torch.where(key[None, :n] <= last[:, None], q @ k[:n].t(), -math.inf)
                norm = z.logsumexp(dim=1)
                lse[head, s["qs"][i] + part] = norm
                out[head, s["qs"][i] + part] = z.sub_(norm[:, None]).exp_() @ v[:n]
    return out, lse


def _pairs(case):
    """Visible (query, key) pairs of one query head."""
    return sum(nq * (nk - nq) + nq * (nq + 1) / 2.0 for nq, nk in _seqs(case))


def _work_attention(case):
    H, G, D, e = case["H"], case["G"], case["D"], _elem(case)
    tq, tk = sum(a for a, _ in _seqs(case)), sum(b for _, b in _seqs(case))
    return {"bytes": 2 * tq * H * G * D * e + 2 * tk * H * D * e + 4 * tq * H * G, "flops": 4.0 * H * G * D * _pairs(case)}


# ---- the paged cache -------------------------------------------------------------------------------------------------


def _lengths(case):
    """Rows in every head: the eight groups of an arithmetic progression, spread over the heads."""
    return [max(1, case["rows"] * (12 - (5 * h + 3) % 8) // 12) for h in range(case["heads"])]


def _cache(case, g, fill):
    """Pages of a pool, handed out in any order, for every head's rows and ROOM more."""
    n, D, page, dt = case["heads"], case["D"], case["page"], _dtype(case)
    length = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    most = -(-(case["rows"] + ROOM) // page)
    need = (length.long() + ROOM + page - 1) // page
    first = torch.cumsum(need, 0) - need
    n_pages = int(need.sum())
    slot = torch.arange(most, device=DEV)[None, :]
    ids = torch.randperm(n_pages, generator=g, device=DEV)
    table = torch.where(slot < need[:, None], ids[(first[:, None] + slot).clamp_(max=n_pages - 1)], -1).to(torch.int32)
    c = dict(n_pages=n_pages, table=table, length=length, K=torch.zeros(n_pages, page, D, dtype=dt, device=DEV),
             V=torch.zeros(n_pages, page, D, dtype=dt, device=DEV), idx=torch.zeros(n_pages, page, dtype=torch.int32, device=DEV),
             cum=torch.zeros(n_pages, page, dtype=torch.float32, device=DEV))
    if fill:
        step = max(1, (1 << 26) // (most * page * D))
        for a in range(0, n, step):
            b = min(n, a + step)
            k, v, idx, cum = _rows(case, g, b - a, most * page)
            rows = torch.arange(most * page, device=DEV)
            live = rows[None, :] < length[a:b, None]
            at = (table[a:b].long()[:, rows // page] * page + rows % page)[live]
            c["K"].view(-1, D)[at], c["V"].view(-1, D)[at] = k[live], v[live]
            c["idx"].view(-1)[at], c["cum"].view(-1)[at] = idx[live], cum[live]
    return c


def _rows(case, g, n, rows):
    """Keys, values, positions and accumulated weights of n heads: ascending positions, one of eight kept, one row in eight without weight."""
    D, dt = case["D"], _dtype(case)
    f = _factors(g, n, 96, D)
    k = (torch.bmm(torch.randn(n, rows, 96, generator=g, device=DEV), f) + 0.1 * torch.randn(n, rows, D, generator=g, device=DEV)).to(dt)
    v = torch.randn(n, rows, D, generator=g, device=DEV).to(dt)
    idx = 8 * torch.arange(rows, device=DEV)[None, :] + torch.randint(0, 8, (n, rows), generator=g, device=DEV)
    cum = torch.exp(torch.randn(n, rows, generator=g, device=DEV)) / rows
    cum = torch.where(torch.rand(n, rows, generator=g, device=DEV) < 0.125, 0.0, cum)
    return k, v, idx.to(torch.int32), cum


def _with_context(state, case, c):
    if own:
        from paper_2410_03090_amd import binding
        state["ctx"] = binding.Context(0, binding.Context.paged_workspace_bytes(case["heads"], case["G"], case["D"],
                                                                                 c["table"].shape[1] * case["page"]))
        state["cache"] = binding.PagedCache(K=c["K"], V=c["V"], idx=c["idx"], cum=c["cum"], table=c["table"], length=c["length"])
    return state


def _flat(c, page, heads, rows):
    """Pool rows of (head, row) pairs."""
    return c["table"][heads, rows // page].long() * page + rows % page


# append: the dense cache of a prompt, as selection and decode set-up leave it, joins empty pages


def _prepare_append(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c = _cache(case, g, False)
    cap, n, D, dt = case["rows"], case["heads"], case["D"], _dtype(case)
    src = dict(K=torch.zeros(n, cap, D, dtype=dt, device=DEV), V=torch.zeros(n, cap, D, dtype=dt, device=DEV),
               idx=torch.zeros(n, cap, dtype=torch.int32, device=DEV), cum=torch.zeros(n, cap, device=DEV), length=c["length"].clone())
    step = max(1, (1 << 26) // (cap * D))
    for a in range(0, n, step):
        b = min(n, a + step)
        src["K"][a:b], src["V"][a:b], src["idx"][a:b], src["cum"][a:b] = _rows(case, g, b - a, cap)
    return _with_context(dict(case=case, c=c, src=src), case, c)


def _run_append(s):
    c, src, page = s["c"], s["src"], s["case"]["page"]
    c["length"].zero_()                                           # a new prompt: the head's pages hold nothing yet
    if own:
        s["ctx"].paged_append(s["cache"], src["K"], src["V"], src["idx"], cum=src["cum"], rows=src["length"])
    else:
        cap = src["K"].shape[1]
        row = torch.arange(cap, device=DEV)[None, :].expand(s["case"]["heads"], cap)
        heads, rows = torch.nonzero(row < src["length"][:, None], as_tuple=True)
        at = _flat(c, page, heads, c["length"][heads] + rows)
        for name in ("K", "V", "idx", "cum"):
            c[name].view(-1, *c[name].shape[2:])[at] = src[name][heads, rows]
        c["length"] += src["length"]
    return _bits(c["K"]), _bits(c["V"]), c["idx"], _bits(c["cum"]), c["length"]


def _work_append(case):
    rows, e = sum(_lengths(case)), _elem(case)
    return {"bytes": 2 * rows * (2 * case["D"] * e + 8), "flops": 0.0}


# step: one generated token


def _prepare_step(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, G, D, dt = case["heads"], case["G"], case["D"], _dtype(case)
    c = _cache(case, g, True)
    rand = lambda *sh: torch.randn(*sh, generator=g, device=DEV)  # noqa: E731
    ring = min(RING, max(2, (1 << 28) // (n * (G + 2) * D)))
    state = dict(case=case, c=c, t=0, start=c["length"].clone(), q=(0.7 * rand(ring, n, G, D)).to(dt), k=rand(ring, n, D).to(dt),
                 v=rand(ring, n, D).to(dt), pos=[torch.full((n,), 8 * (case["rows"] + ROOM) + t, dtype=torch.int32, device=DEV) for t in range(ROOM)],
                 out=torch.empty(n, G, D, dtype=torch.float32, device=DEV))
    return _with_context(state, case, c)


def _step_plain(s, q, k, v, pos):
    c, case = s["c"], s["case"]
    n, G, D, page = case["heads"], case["G"], case["D"], case["page"]
    every = torch.arange(n, device=DEV)
    at = _flat(c, page, every, c["length"].long())
    c["K"].view(-1, D)[at], c["V"].view(-1, D)[at] = k, v
    c["idx"].view(-1)[at], c["cum"].view(-1)[at] = pos, 0.0
    c["length"] += 1
    rows = torch.arange(c["table"].shape[1] * page, device=DEV)
    step = max(1, (1 << 28) // (rows.numel() * D))
    for a in range(0, n, step):
        b = min(n, a + step)
        live = rows[None, :] < c["length"][a:b, None]
        at = c["table"][a:b].long().clamp(min=0)[:, rows // page] * page + rows % page
        kk, vv = c["K"].view(-1, D)[at].float(), c["V"].view(-1, D)[at].float()
        logits = torch.matmul(kk, q[a:b].float().transpose(1, 2).contiguous()) / math.sqrt(D)           # [heads, rows, G]
        p = torch.softmax(logits.masked_fill_(~live[:, :, None], float("-inf")), dim=1)
        s["out"][a:b] = torch.matmul(p.transpose(1, 2).contiguous(), vv)
        c["cum"].view(-1)[at[live]] += p.sum(dim=2)[live]


def _run_step(s):
    c, t = s["c"], s["t"]
    s["t"] = t + 1
    if t > 0 and t % ROOM == 0:
        c["length"].copy_(s["start"])                             # the rows behind the budgets left
    r, pos = t % s["q"].shape[0], s["pos"][t % ROOM]
    if own:
        s["ctx"].paged_step(s["cache"], s["q"][r], s["k"][r], s["v"][r], pos, out=s["out"])
    else:
        _step_plain(s, s["q"][r], s["k"][r], s["v"][r], pos)
    return s["out"], c["cum"], _bits(c["K"]), _bits(c["V"]), c["idx"], c["length"]


def _exact_step(case, seed):
    s = _prepare_step(case, seed)
    c, G, D, page = s["c"], case["G"], case["D"], case["page"]
    out = torch.empty(case["heads"], G, D, dtype=torch.float64, device=DEV)
    cum = c["cum"].double()
    lengths = _lengths(case)
    for h in range(case["heads"]):
        pages = c["table"][h, :-(-(lengths[h] + 1) // page)].long()
        keys, values = c["K"][pages].flatten(0, 1)[:lengths[h] + 1].double(), c["V"][pages].flatten(0, 1)[:lengths[h] + 1].double()
        keys[lengths[h]], values[lengths[h]] = s["k"][0, h], s["v"][0, h]
        z = s["q"][0, h].double() @ keys.t() * D ** -0.5
        weight = (z - z.logsumexp(dim=1, keepdim=True)).exp()
        out[h] = weight @ values
        grown = cum[pages].flatten()
        grown[lengths[h]] = 0.0
        grown[:lengths[h] + 1] += weight.sum(dim=0)
        cum[pages] = grown.view(-1, page)
    return out, cum, None, None, None, None


def _work_step(case):
    rows, n, e = sum(_lengths(case)) + case["heads"], case["heads"], _elem(case)
    new = n * ((2 + case["G"]) * case["D"] * e + 4 * case["G"] * case["D"])
    return {"bytes": rows * (2 * case["D"] * e + 8) + new, "flops": 4.0 * rows * case["G"] * case["D"]}


# evict: budgets are kept again


def _prepare_evict(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c = _cache(case, g, True)
    # one buffer for what an eviction reads and rewrites besides the rows, so that one copy brings it back
    n, rows = case["heads"], c["idx"].numel()
    small = torch.empty(2 * rows + n, dtype=torch.int32, device=DEV)
    small[:rows], small[rows:2 * rows], small[2 * rows:] = c["idx"].view(-1), _bits(c["cum"]).view(-1), c["length"]
    c["idx"], c["cum"] = small[:rows].view(c["idx"].shape), small[rows:2 * rows].view(torch.float32).view(c["cum"].shape)
    c["length"] = small[2 * rows:]
    budget = (c["length"] * case["keep"]).to(torch.int32).clamp_(min=1)
    pos = torch.full((n,), 8 * case["rows"], dtype=torch.int32, device=DEV)
    return _with_context(dict(case=case, c=c, small=small, start=small.clone(), budget=budget, pos=pos, w=32), case, c)


def _evict_plain(s):
    c, page, D, n = s["c"], s["case"]["page"], s["case"]["D"], s["case"]["heads"]
    rows = torch.arange(c["table"].shape[1] * page, device=DEV)
    step = max(1, (1 << 25) // rows.numel())
    for a in range(0, n, step):
        b = min(n, a + step)
        length = c["length"][a:b].clone()
        live = rows[None, :] < length[:, None]
        at = c["table"][a:b].long().clamp(min=0)[:, rows // page] * page + rows % page
        idx, cum = c["idx"].view(-1)[at], c["cum"].view(-1)[at]
        old = live & (idx <= (s["pos"][a:b] - s["w"])[:, None])
        drop = torch.minimum((length - s["budget"][a:b].clamp(min=s["w"])).clamp(min=0).long(), old.sum(dim=1))
        order = torch.argsort(idx, dim=1, stable=True)
        key = torch.where(old, cum, float("inf"))
        order = order.gather(1, torch.argsort(key.gather(1, order), dim=1, stable=True))
        rank = torch.empty_like(order).scatter_(1, order, rows[None, :].expand_as(order))
        leaves = rank < drop[:, None]
        left = length.long() - drop
        hole = torch.nonzero(leaves & (rows[None, :] < left[:, None]), as_tuple=True)
        mover = torch.nonzero(live & ~leaves & (rows[None, :] >= left[:, None]), as_tuple=True)
        src, dst = at[mover], at[hole]                            # row by row, head by head: as many of one as of the other
        for name in ("K", "V", "idx", "cum"):
            flat = c[name].view(-1, *c[name].shape[2:])
            flat[dst] = flat[src]
        c["length"][a:b] = left.to(torch.int32)


def _run_evict(s):
    c = s["c"]
    s["small"].copy_(s["start"])                                  # the cache is over its budgets again
    if own:
        s["ctx"].paged_evict(s["cache"], s["budget"], s["pos"], s["w"])
    else:
        _evict_plain(s)
    return _bits(c["K"]), _bits(c["V"]), c["idx"], _bits(c["cum"]), c["length"]


def _work_evict(case):
    rows, e, keep = sum(_lengths(case)), _elem(case), case["keep"]
    return {"bytes": rows * 8 + rows * keep * (1.0 - keep) * 2 * (2 * case["D"] * e + 8), "flops": 0.0}


_PREPARE = dict(attention=_prepare_attention, append=_prepare_append, step=_prepare_step, evict=_prepare_evict)
_RUN = dict(attention=_run_attention, append=_run_append, step=_run_step, evict=_run_evict)
_WORK = dict(attention=_work_attention, append=_work_append, step=_work_step, evict=_work_evict)
_EXACT = dict(attention=_exact_attention, step=_exact_step)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed)


def run(state):
    return _RUN[state["case"]["kind"]](state)


def work(case):
    return _WORK[case["kind"]](case)


def exact(case, seed):
    """Appending and evicting copy rows: they have no computed numbers."""
    make = _EXACT.get(case["kind"])
    return make(case, seed) if make else None
