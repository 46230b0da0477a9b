"""Cases and plain forms of the paged token memory and of attention with a window.

Token histories that branch and age (hypotheses of tracked objects, streams of
frames) are kept in pages of 8-bit numbers.  A page holds `page` places of one
sequence; 16 places of a page and key head are a block with one power of two for
its keys and one for its values.  Operators:

    pages    which pages a sequence has: a fork takes over its parent's pages,
             drops those behind the window and counts references, an extension
             gives pages to new tokens and lists the shared pages to copy, a
             compaction moves the pages in use to the pool's front; the listed
             pages are copied (rtcc_pages_fork, rtcc_pages_extend,
             rtcc_pages_compact, rtcc_pages_copy);
    write    keys and values of new tokens rounded to 8 bits in their blocks
             (rtcc_pages_write);
    attend   attention over the pages (rtcc_pages_attention);
    window   attention over the 16-bit memory with a sliding window and a few
             first tokens that stay visible (rtcc_memory_window_attention).

run() computes a case by elementary torch operations in 32 bits, or, where
`own` is set, by the framework's calls.  exact() is the definition in 64 bits.
8-bit numbers are returned as float8 values beside their exponents.
"""
import math
import random

import torch

own = False

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 16
E_MIN, E_MAX = -120, 120


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # eight hypotheses of one object resampled, a new token each (latency)
        dict(name="branch_few", op="pages", kind="branch", seqs=8, parents=8, k=300, new=1, window=0, sinks=0, page=64,
             pages=256, kv=4, dim=64),
        # 2048 histories resampled to 1700 parents, up to 37 new tokens each, old pages dropped behind a window
        dict(name="branch_many", op="pages", kind="branch", seqs=2048, parents=1700, k=777, new=37, window=200, sinks=4,
             page=64, pages=16384, kv=4, dim=64),
        # a small pool after a third of its pages were freed
        dict(name="compact_few", op="pages", kind="compact", seqs=7, page=32, pages=500, live=0.6, table=61, kv=3, dim=80),
        # a large pool, half of it free, scattered
        dict(name="compact_many", op="pages", kind="compact", seqs=512, page=64, pages=8192, live=0.5, table=32, kv=8,
             dim=128),
        # a decision step: one token each of 61 tracked requests, blocks partly filled
        dict(name="write_step", op="write", seqs=61, new=1, k=2000, kv=8, dim=128, page=64, dtype="bf16", packed=True),
        # ragged chunks of nine sequences behind their histories, odd sizes
        dict(name="write_chunk", op="write", seqs=9, new=8000, k=333, kv=8, dim=112, page=128, dtype="fp16", packed=False),
        # one query over a short history: the latency of a call
        dict(name="attend_token", op="attend", seqs=1, q=1, k=4097, window=0, sinks=0, heads=6, kv=6, dim=64, page=32,
             dtype="fp16", cap=0.0, ragged=False),
        # a decision step of 61 sequences with ragged histories, grouped heads, capped scores
        dict(name="attend_step", op="attend", seqs=61, q=1, k=16384, window=0, sinks=0, heads=32, kv=8, dim=128, page=64,
             dtype="bf16", cap=30.0, ragged=True),
        # ragged chunks of five prompts through a window of their histories
        dict(name="attend_chunk", op="attend", seqs=5, q=2100, k=9000, window=4000, sinks=16, heads=16, kv=4, dim=128,
             page=128, dtype="bf16", cap=0.0, ragged=True),
        # one query, a short window (latency)
        dict(name="window_token", op="window", seqs=1, q=1, k=50000, window=1000, sinks=4, heads=12, kv=4, dim=80,
             dtype="fp16", cap=0.0, ragged=False, gap=0),
        # the 61 sequences of a decision step, each over the last 5000 of its tokens and the first 16
        dict(name="window_step", op="window", seqs=61, q=1, k=16384, window=5000, sinks=16, heads=32, kv=8, dim=128,
             dtype="bf16", cap=30.0, ragged=True, gap=40),
        # packed ragged sequences, every token over the last 700
        dict(name="window_packed", op="window", seqs=5, q=6000, k=6000, window=700, sinks=8, heads=16, kv=4, dim=128,
             dtype="bf16", cap=0.0, ragged=True, gap=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "pages", "write", "attend", "attend", "attend", "window", "window", "window"])
    kv = rng.choice([1, 2, 3, 4, 5, 6, 8])
    group = rng.choice([1, 1, 2, 3, 4, 8]) if kv <= 4 else rng.choice([1, 1, 2, 4])
    page = rng.choice([32, 64, 64, 128])
    dim8 = rng.choice([16, 32, 48, 64, 64, 64, 80, 96, 112, 128, 128, 128])
    if op == "pages":
        kv = min(kv, 4)
        if rng.random() < 0.5:
            c = dict(op=op, kind="branch", seqs=_log(rng, 1, 2048), parents=_log(rng, 1, 2048), k=_log(rng, 1, 777),
                     new=_log(rng, 1, 37), window=0, sinks=0, page=page, pages=0, kv=kv, dim=min(dim8, 64))
            if rng.random() < 0.5:
                c.update(window=_log(rng, 1, 500), sinks=rng.randint(0, 40))
            # room for most, not always all, of what may be asked for
            per = -(-(c["k"] + c["new"]) // page)
            c["pages"] = max(4, min(16384 * 64 // page, int(per * (c["seqs"] + c["parents"]) * rng.uniform(0.6, 1.2))))
            return c
        pages = _log(rng, 10, 8192 * 64 // page)
        return dict(op=op, kind="compact", seqs=_log(rng, 1, 512), page=page, pages=pages, live=rng.uniform(0.05, 0.95),
                    table=_log(rng, 1, 64), kv=kv, dim=dim8)
    dtype = rng.choice(["fp16", "bf16"])
    if op == "write":
        seqs = _log(rng, 1, 64)
        return dict(op=op, seqs=seqs, new=_log(rng, 1, max(1, min(8000, 9 * 8000 // seqs))), k=_log(rng, 1, 2000), kv=kv,
                    dim=dim8, page=page, dtype=dtype, packed=rng.random() < 0.5)
    dim = dim8 if op == "attend" else rng.choice([16, 32, 40, 64, 64, 64, 72, 80, 96, 104, 128, 128, 128])
    c = dict(op=op, seqs=1, q=1, k=1, window=0, sinks=0, heads=kv * group, kv=kv, dim=dim, dtype=dtype,
             cap=rng.choice([0.0, 0.0, 20.0, 30.0, 50.0]), ragged=rng.random() < 0.7)
    c.update(dict(page=page) if op == "attend" else dict(gap=rng.randint(0, 50)))
    kind = rng.choice(["step", "step", "chunk", "packed"])
    if kind == "step":
        c.update(seqs=_log(rng, 1, 80))
        c.update(k=min(60000, _log(rng, 1, max(1, 61 * 16384 * 8 * 128 // (c["seqs"] * kv * group * dim)))))
    elif kind == "chunk":
        c.update(seqs=_log(rng, 1, 16), q=_log(rng, 2, 100), k=_log(rng, 100, 10000))
    else:
        c.update(seqs=_log(rng, 1, 6), q=_log(rng, 64, 2500))
        c.update(k=c["q"] + rng.choice([0, 0, rng.randint(0, 3000)]))
    if op == "window" or rng.random() < 0.5:
        c.update(window=_log(rng, 1, max(2, c["k"])), sinks=rng.choice([0, 1, 4, 16, rng.randint(0, 200)]))
    # no more score elements than the largest listed cases
    while c["heads"] * c["seqs"] * c["q"] * c["k"] > 16 * 5 * 2100 * 9000 and c["q"] > 1:
        c["q"] = (c["q"] + 1) // 2
    return c


# ---------------------------------------------------------------------------
# sizes of a case (the sequences' lengths come from the case, values from the seed)
# ---------------------------------------------------------------------------

def _spans(c):
    """Per sequence: tokens, and keys with those tokens; ragged ones have from half of
    the tokens and a 16th of the keys up, the first sequence the most."""
    rng = random.Random("%d %d %d" % (c["seqs"], c["q"], c["k"]))
    n, held = [], []
    for i in range(c["seqs"]):
        q, k = c["q"], max(c["k"], c["q"])
        if c["ragged"] and i:
            q = rng.randint((c["q"] + 1) // 2, c["q"])
            k = max(q, rng.randint(max(1, c["k"] // 16), c["k"]))
        n.append(q)
        held.append(k)
    return n, held


def _write_spans(c):
    rng = random.Random("%d %d" % (c["seqs"], c["new"]))
    new = [rng.randint((c["new"] + 1) // 2, c["new"]) if i else c["new"] for i in range(c["seqs"])]
    held = [rng.randint(0, c["k"]) for i in range(c["seqs"])]
    return new, held


def _visible(c):
    """Visible (query, key) pairs of one head, and keys that any token sees."""
    n, held = _spans(c)
    w, z = c["window"], c["sinks"]
    pairs = keys = 0
    for q, k in zip(n, held):
        first = k - q
        for i in range(q):
            end = first + i + 1
            lo = max(0, end - w) if w else 0
            pairs += end - lo + min(z if w else 0, lo)
        lo = max(0, first + 1 - w) if w else 0
        keys += k - lo + min(z if w else 0, lo)
    return pairs, keys


def _row_bytes(c):
    return 2 * c["kv"] * c["dim"]                        # keys and values of a place, 8 bits each


def work(c):
    if c["op"] == "pages" and c["kind"] == "branch":
        per = -(-(c["k"] + c["new"]) // c["page"])
        # tables read and written, references, and about half a page of every second sequence copied
        table = 4 * per * (c["seqs"] + min(c["seqs"], c["parents"]))
        return {"bytes": table + 4 * c["pages"] + 28 * c["seqs"] + c["seqs"] // 2 * (c["page"] // 2) * _row_bytes(c) * 2,
                "flops": 0}
    if c["op"] == "pages":
        moves = int(c["pages"] * c["live"] * (1 - c["live"]))
        return {"bytes": 8 * c["seqs"] * c["table"] + 8 * c["pages"] + 8 * moves + moves * c["page"] * _row_bytes(c) * 2,
                "flops": 0}
    if c["op"] == "write":
        new, _ = _write_spans(c)
        return {"bytes": sum(new) * c["kv"] * c["dim"] * 2 * 3 + sum(new) // 16 * c["kv"] * 2, "flops": 0}
    pairs, keys = _visible(c)
    tokens = sum(_spans(c)[0])
    each = (2 * c["dim"] + 2 / BLOCK) if c["op"] == "attend" else 4 * c["dim"]
    return {"bytes": 4 * tokens * c["heads"] * c["dim"] + int(keys * c["kv"] * each) + 4 * tokens * c["heads"],
            "flops": pairs * c["heads"] * 4 * c["dim"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _full(n, v=-1):
    return torch.full(n if isinstance(n, tuple) else (n,), v, dtype=torch.int32, device="cuda")


def _need(top):
    """Least e with top <= 448 * 2^e, from E_MIN to E_MAX."""
    m, x = torch.frexp(top)                              # top = m 2^x, m in [0.5, 1)
    e = x - 9 + (m > 0.875).to(x.dtype)
    return torch.where(top > 0, e, E_MIN).clamp(E_MIN, E_MAX)


def _pool(g, c, pages):
    """A pool as earlier writes left it: codes uint8 [pages][kv][page][dim] of keys and values, exponents
    int8 [pages][kv][page / 16][2]; heads of unlike scale, some tokens far larger than the rest."""
    kv, pr, d = c["kv"], c["page"], c["dim"]
    codes = [torch.empty(pages, kv, pr, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = torch.empty(pages, kv, pr // BLOCK, 2, dtype=torch.int8, device="cuda")
    step = max(1, (1 << 26) // (kv * pr * d))
    for which in range(2):
        size = 0.5 + 1.0 * torch.rand(kv, 1, 1, generator=g, device="cuda")
        for a in range(0, pages, step):
            n = min(step, pages - a)
            x = torch.randn(n, kv, pr, d, generator=g, device="cuda") * size
            x *= torch.where(torch.rand(n, kv, pr, 1, generator=g, device="cuda") < 0.02, 3.0, 1.0)
            x = x.view(n, kv, pr // BLOCK, BLOCK * d)
            e = _need(x.abs().amax(-1))
            scales[a:a + n, ..., which] = e.to(torch.int8)
            x = torch.ldexp(x, -e[..., None]).view(n, kv, pr, d)
            codes[which][a:a + n] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes[0], codes[1], scales


def prepare(case, seed):
    return {"pages": _prepare_pages, "write": _prepare_write, "attend": _prepare_attend,
            "window": _prepare_window}[case["op"]](case, seed)


def _prepare_pages(c, seed):
    g = _gen(seed)
    kp, vp, scales = _pool(g, c, c["pages"])
    s = dict(case=c, k_pages=kp, v_pages=vp, scales=scales, space=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    rand = lambda n: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    n, pages = c["seqs"], c["pages"]
    if c["kind"] == "compact":
        # live pages scattered; entries name them, some shared, the rest of the table empty
        live = torch.nonzero(rand(pages) < c["live"])[:, 0]
        cells = n * c["table"]
        table = _full(cells)
        if live.numel():
            at = torch.randperm(cells, generator=g, device="cuda")
            used = int(cells * 0.8)
            pick = live[(torch.arange(used, device="cuda") * 0.9).long() % live.numel()]
            table[at[:used]] = pick.int()
        refs = torch.bincount(table[table >= 0].long(), minlength=pages).int()
        return dict(s, table=table.view(n, c["table"]), refs=refs, table_out=_full((n, c["table"])), refs_out=_full(pages),
                    src=_full(pages), dst=_full(pages), count=_full(1))
    # histories of up to k places on pages of their own, of a pool with room left for their children
    per = -(-(c["k"] + c["new"]) // c["page"])
    length = (c["k"] * (0.5 + 0.5 * rand(c["parents"]))).int().clamp(min=1)
    want = (length + c["page"] - 1) // c["page"]
    order = torch.randperm(pages, generator=g, device="cuda").int()
    first = torch.cumsum(want, 0) - want
    at = first[:, None] + torch.arange(per, device="cuda")
    have = (torch.arange(per, device="cuda") < want[:, None]) & (at < pages * 7 // 10)
    table = torch.where(have, order[at.clamp(max=pages - 1)], -1).int()
    length = torch.minimum(length, have.sum(1).int() * c["page"])
    # resampling: most continue one of a few parents; one in 20 is given up, one in 10 loses its last tokens
    parent = (c["parents"] * rand(n) ** 2).int().clamp(max=c["parents"] - 1)
    parent = torch.where(rand(n) < 0.05, -1, parent).int()
    keep = torch.where(rand(n) < 0.1, (c["k"] * rand(n)).int(), 1 << 30).int()
    new = (rand(n) * (c["new"] + 1)).int().clamp(max=c["new"])
    return dict(s, parent=parent, keep=keep, new=new, length=length, table=table.contiguous(), held=_full(n),
                table_out=_full((n, per)), refs=_full(pages), length_out=_full(n), src=_full(n), dst=_full(n), rows=_full(n),
                short=_full(1))


def _chain(g, lengths, page, spare=3):
    """A table for sequences of these lengths on shuffled pages, and the pages there are."""
    per = max(1, max(-(-v // page) for v in lengths))
    total = sum(-(-v // page) for v in lengths) + spare
    order = torch.randperm(total, generator=g, device="cuda").int()
    want = _i32([-(-v // page) for v in lengths]).long()
    first = torch.cumsum(want, 0) - want
    at = torch.arange(per, device="cuda")
    table = torch.where(at < want[:, None], order[(first[:, None] + at).clamp(max=total - 1)], -1)
    return table.int().contiguous(), total


def _prepare_write(c, seed):
    g = _gen(seed)
    new, held = _write_spans(c)
    n = sum(new)
    table, pages = _chain(g, [a + b for a, b in zip(new, held)], c["page"])
    kp, vp, scales = _pool(g, c, pages)
    kv, d, dt = c["kv"], c["dim"], DT[c["dtype"]]
    # a projection's output: heads of unlike scale; packed = keys and values of a token in one row
    size = 0.2 + 2 * torch.rand(2, kv, 1, generator=g, device="cuda")
    x = (torch.randn(n, 2, kv, d, generator=g, device="cuda") * size).to(dt)
    k, v = x[:, 0], x[:, 1]
    if not c["packed"]:
        k, v = k.contiguous(), v.contiguous()
    return dict(case=c, k=k, v=v, offsets=_i32([sum(new[:i]) for i in range(len(new) + 1)]), held=_i32(held),
                length=_i32([a + b for a, b in zip(new, held)]), table=table, k_pages=kp, v_pages=vp, scales=scales)


def _prepare_attend(c, seed):
    g = _gen(seed)
    n, held = _spans(c)
    table, pages = _chain(g, held, c["page"])
    kp, vp, scales = _pool(g, c, pages)
    tokens, hq, d, dt = sum(n), c["heads"], c["dim"], DT[c["dtype"]]
    q = (1.2 * torch.randn(tokens, hq, d, generator=g, device="cuda")).to(dt)
    if c["window"]:
        # what lies behind every window, past the sinks, has been freed
        start = _i32([h - m for m, h in zip(n, held)])[:, None]
        at = torch.arange(table.shape[1], device="cuda") * c["page"]
        gone = (at >= c["sinks"]) & (at + c["page"] - 1 <= start - c["window"])
        table = torch.where(gone, -1, table).int().contiguous()
    rows = 64 + max(held) if not c["window"] else min(64 + max(held), c["sinks"] + c["window"] + max(n) + 256)
    space = (64 << 20) + len(n) * rows * c["kv"] * d * 4
    return dict(case=c, q=q, offsets=_i32([sum(n[:i]) for i in range(len(n) + 1)]), length=_i32(held),
                start=_i32([h - m for m, h in zip(n, held)]), table=table, k_pages=kp, v_pages=vp, scales=scales,
                max_q=max(n), max_k=max(held), out=torch.zeros(tokens, hq, d, dtype=dt, device="cuda"),
                lse=torch.zeros(tokens, hq, device="cuda"), space=torch.empty(space, dtype=torch.uint8, device="cuda"))


def _prepare_window(c, seed):
    g = _gen(seed)
    n, held = _spans(c)
    hq, hk, d, dt, tokens = c["heads"], c["kv"], c["dim"], DT[c["dtype"]], sum(n)
    begin, at = [], c["gap"]
    for h in held:
        begin.append(at)
        at += h + c["gap"]
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    q = (1.5 * rand(tokens, hq, d)).to(dt)
    k, v = rand(at, hk, d).to(dt), rand(at, hk, d).to(dt)
    return dict(case=c, q=q, k=k, v=v, begin=_i32(begin), end=_i32([b + h for b, h in zip(begin, held)]),
                offsets=_i32([sum(n[:i]) for i in range(len(n) + 1)]), start=_i32([h - m for m, h in zip(n, held)]),
                max_q=max(n), max_k=max(held), out=torch.zeros(tokens, hq, d, dtype=dt, device="cuda"),
                lse=torch.zeros(tokens, hq, device="cuda"),
                space=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return {"pages": _own_pages, "write": _own_write, "attend": _own_attend, "window": _own_window}[c["op"]](s, c)
    return {"pages": _plain_pages, "write": _plain_write, "attend": _plain_attend, "window": _plain_window}[c["op"]](s, c)


def _f8(s):
    return [s["k_pages"].view(torch.float8_e4m3fn), s["v_pages"].view(torch.float8_e4m3fn), s["scales"]]


def _config(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    table = s["table_out"] if c["op"] == "pages" else s["table"]
    return R.page_config(c["kv"], c["dim"], c["page"], s["k_pages"].shape[0], table.shape[0], table.shape[1])


def _own_pages(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    stream = torch.cuda.current_stream().cuda_stream
    p = {n: t.data_ptr() for n, t in s.items() if isinstance(t, torch.Tensor)}
    cfg = _config(s, c)
    pool = (p["k_pages"], p["v_pages"], p["scales"])
    if c["kind"] == "compact":
        R.check(R.rtcc_pages_compact(cfg, p["table"], p["refs"], p["table_out"], p["refs_out"], p["src"], p["dst"],
                                     p["count"], p["space"], s["space"].numel(), stream))
        R.check(R.rtcc_pages_copy(cfg, c["pages"], p["count"], p["src"], p["dst"], None, *pool, c["pages"], *pool, stream))
        return [s["table_out"], s["refs_out"], s["src"], s["dst"], s["count"]] + _f8(s)
    R.check(R.rtcc_pages_fork(cfg, c["parents"], p["parent"], p["keep"], c["window"], c["sinks"], p["length"], p["table"],
                              p["held"], p["table_out"], p["refs"], stream))
    R.check(R.rtcc_pages_extend(cfg, p["new"], p["held"], p["table_out"], p["refs"], p["length_out"], p["src"], p["dst"],
                                p["rows"], p["short"], p["space"], s["space"].numel(), stream))
    R.check(R.rtcc_pages_copy(cfg, c["seqs"], None, p["src"], p["dst"], p["rows"], *pool, c["pages"], *pool, stream))
    return [s["held"], s["table_out"], s["refs"], s["length_out"], s["src"], s["dst"], s["rows"], s["short"]] + _f8(s)


def _plain_copy(s, c, src, dst, rows):
    """Rows [0, rows) of every listed page, and the exponents of the blocks they begin in."""
    live = torch.nonzero(src >= 0)[:, 0]
    a, b = src[live].long(), dst[live].long()
    n = rows[live].long() if rows is not None else torch.full_like(a, c["page"])
    r = torch.arange(c["page"], device="cuda")
    pick = (r < n[:, None])[:, None, :, None]
    for p in (s["k_pages"], s["v_pages"]):
        p[b] = torch.where(pick, p[a], p[b])
    blocks = (r[::BLOCK] < n[:, None])[:, None, :, None]
    s["scales"][b] = torch.where(blocks, s["scales"][a], s["scales"][b])


def _plain_pages(s, c):
    if c["kind"] == "compact":
        pages = c["pages"]
        live = s["refs"] > 0
        index = torch.arange(pages, device="cuda")
        n = live.sum()
        order = torch.argsort(torch.where(live & (index >= n), index, pages + index))       # live pages behind n first
        holes = torch.argsort(torch.where(~live & (index < n), index, pages + index))
        count = (live & (index >= n)).sum()
        on = index < count
        src, dst = torch.where(on, order, -1), torch.where(on, holes, -1)
        to = index.clone()
        to[order] = torch.where(on, holes, order)
        table = torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], -1)
        refs = torch.zeros_like(s["refs"])
        refs[to[live]] = s["refs"][live]
        _plain_copy(s, c, src, dst, None)
        return [table.int(), refs, src.int(), dst.int(), count.int()[None]] + _f8(s)
    pr, per, pages = c["page"], s["table"].shape[1], c["pages"]
    parent = s["parent"].long()
    ok = parent >= 0
    length = torch.minimum(torch.where(ok, s["length"][parent.clamp(min=0)], 0), s["keep"]).clamp(0, per * pr)
    at = torch.arange(per, device="cuda") * pr
    table = torch.where(ok[:, None] & (at < length[:, None]), s["table"][parent.clamp(min=0)], -1).long()
    if c["window"]:
        gone = (at >= c["sinks"]) & (at + pr - 1 <= (length - c["window"])[:, None])
        table = torch.where(gone, -1, table)
    refs = torch.bincount(table.flatten() + 1, minlength=pages + 1)[1:]
    held = length.clone()
    # what every place of the tables asks for: the shared last page, and pages for the new places
    end = torch.minimum(held + s["new"], torch.full_like(held, per * pr))
    last = (held // pr).clamp(max=per - 1).long()[:, None]
    mine = table.gather(1, last)[:, 0]
    partly = (end > held) & (held % pr != 0)
    shared = partly & (mine >= 0) & (refs[mine.clamp(min=0)] > 1)
    fresh = partly & (mine < 0)
    wants = (at >= held[:, None]) & (at < end[:, None])
    wants.scatter_(1, last, (wants.gather(1, last)[:, 0] | shared | fresh)[:, None])
    rank = (torch.cumsum(wants.flatten().long(), 0) - 1).view_as(wants)
    free = torch.argsort(torch.where(refs == 0, 0, 1), stable=True)
    n_free, asked = (refs == 0).sum(), wants.sum()
    got = wants & (rank < n_free)
    given = free[rank.clamp(0, pages - 1)]
    # a shared page that has no substitute stays, and its sequence as it is
    lost = wants & ~got
    stay = torch.zeros_like(wants).scatter_(1, last, shared[:, None]) & lost
    copied = shared & got.gather(1, last)[:, 0]
    src = torch.where(copied, mine, -1)
    table = torch.where(got, given, torch.where(lost & ~stay, -1, table))
    dst = torch.where(copied, table.gather(1, last)[:, 0], -1)
    rows = torch.where(copied, held % pr, 0)
    refs = refs.scatter_add(0, given[got], torch.ones_like(given[got]))
    refs = refs.scatter_add(0, mine[copied], -torch.ones_like(mine[copied]))
    gap = torch.where(lost, at, per * pr).amin(1)
    out = torch.maximum(torch.minimum(end, gap.int()), held)
    short = (asked - got.sum()).int()[None]
    _plain_copy(s, c, src, dst, rows)
    return [held, table.int(), refs.int(), out, src.int(), dst.int(), rows.int(), short] + _f8(s)


def _own_write(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    k, v = s["k"], s["v"]
    new = R.write_config(R.BF16 if c["dtype"] == "bf16" else R.FP16, k.shape[0], c["new"], k.stride()[:2], v.stride()[:2])
    R.check(R.rtcc_pages_write(_config(s, c), new, k.data_ptr(), v.data_ptr(), s["offsets"].data_ptr(),
                               s["held"].data_ptr(), s["length"].data_ptr(), s["table"].data_ptr(),
                               s["k_pages"].data_ptr(), s["v_pages"].data_ptr(), s["scales"].data_ptr(),
                               torch.cuda.current_stream().cuda_stream))
    return _f8(s)


def _plain_write(s, c):
    pr, nb, kv, d = c["page"], c["page"] // BLOCK, c["kv"], c["dim"]
    off, held = s["offsets"].long(), s["held"].long()
    at = torch.arange(s["k"].shape[0], device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), at, right=True)
    place = held[seq] + at - off[seq]
    page = s["table"][seq, place // pr].long()
    block = page * nb + place % pr // BLOCK                              # of all blocks of the pool
    # the block in which a sequence's new tokens begin, and the rows that it holds already
    has = held % BLOCK != 0
    old_page = s["table"].gather(1, (held // pr)[:, None])[has, 0].long()
    old_block, old_rows = old_page * nb + held[has] % pr // BLOCK, held[has] % BLOCK
    pages = s["k_pages"].shape[0]
    for which, x, codes in ((0, s["k"], s["k_pages"]), (1, s["v"], s["v_pages"])):
        x = x.float()
        fine = torch.isfinite(x)
        top = torch.where(fine, x.abs(), 0.0).amax(-1)                   # [tokens, kv]
        most = torch.zeros(pages * nb, kv, device="cuda").scatter_reduce_(0, block[:, None].expand(-1, kv), top, "amax")
        e = _need(most)                                                  # [blocks of the pool, kv]
        was = s["scales"][..., which].permute(0, 2, 1).reshape(pages * nb, kv).int()
        touched = torch.zeros(pages * nb, dtype=torch.bool, device="cuda").index_fill_(0, block, True)
        holds = torch.zeros_like(touched).index_fill_(0, old_block, True)
        e = torch.where(holds[:, None], torch.maximum(e, was), e)
        e = torch.where(touched[:, None], e, was)
        s["scales"][..., which] = e.view(pages, nb, kv).permute(0, 2, 1).to(torch.int8)
        # rows held so far, rounded again where the exponent rose
        rows = codes.view(pages, kv, nb, BLOCK, d).permute(0, 2, 1, 3, 4)
        b = (old_block // nb, old_block % nb)
        val = rows[b]                                                    # [seqs, kv, 16, d]
        again = torch.ldexp(val.view(torch.float8_e4m3fn).float(), (was - e)[old_block][..., None, None])
        again = again.to(torch.float8_e4m3fn).view(torch.uint8)
        keep = (torch.arange(BLOCK, device="cuda") < old_rows[:, None])[:, None, :, None]
        rows[b] = torch.where(keep & (was < e)[old_block][..., None, None], again, val)
        y = torch.ldexp(torch.where(fine, x, math.nan), -e[block][..., None]).to(torch.float8_e4m3fn)
        codes[page, :, place % pr] = y.view(torch.uint8)
    return _f8(s)


def _own_attend(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    q, out = s["q"], s["out"]
    cfg = R.page_attn_config(c["heads"], R.BF16 if c["dtype"] == "bf16" else R.FP16, q.shape[0], q.stride()[:2],
                             out.stride()[:2], s["max_q"], s["max_k"], causal=True, window=c["window"], sinks=c["sinks"],
                             scale=1 / math.sqrt(c["dim"]), cap=c["cap"])
    R.check(R.rtcc_pages_attention(_config(s, c), cfg, q.data_ptr(), s["offsets"].data_ptr(), s["start"].data_ptr(),
                                   s["length"].data_ptr(), None, s["table"].data_ptr(), s["k_pages"].data_ptr(),
                                   s["v_pages"].data_ptr(), s["scales"].data_ptr(), out.data_ptr(), s["lse"].data_ptr(),
                                   s["space"].data_ptr(), s["space"].numel(), torch.cuda.current_stream().cuda_stream))
    return [out, s["lse"]]


def _own_window(s, c):
    from paper_2608_08330_gb300 import rtcc as R
    q, k, v, out = s["q"], s["k"], s["v"], s["out"]
    cfg = R.attn_config(c["heads"], c["kv"], c["dim"], R.BF16 if c["dtype"] == "bf16" else R.FP16, q.shape[0], k.shape[0],
                        q.stride()[:2], k.stride()[:2], v.stride()[:2], out.stride()[:2], c["seqs"], s["max_q"],
                        s["max_k"], causal=True, scale=1 / math.sqrt(c["dim"]), cap=c["cap"],
                        q_start=s["start"].data_ptr())
    R.check(R.rtcc_memory_window_attention(cfg, c["window"], c["sinks"], q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                           s["offsets"].data_ptr(), s["begin"].data_ptr(), s["end"].data_ptr(), None, None,
                                           None, None, None, out.data_ptr(), s["lse"].data_ptr(), s["space"].data_ptr(),
                                           s["space"].numel(), torch.cuda.current_stream().cuda_stream))
    return [out, s["lse"]]


def _plain_values(s, codes, which, pages, rows):
    """Keys or values of the given pages' rows [B, L, kv, d] in 32 bits, from codes and exponents."""
    x = codes[pages, :, rows].view(torch.float8_e4m3fn).float()
    e = s["scales"][..., which][pages, :, rows // BLOCK].int()
    return torch.ldexp(x, e[..., None])


def _plain_attend(s, c):
    at = torch.arange(s["max_k"], device="cuda")
    page = s["table"][:, at // c["page"]].long()                         # [B, L]
    pages, rows = page.clamp(min=0), (at % c["page"]).expand_as(page)
    k = _plain_values(s, s["k_pages"], 0, pages, rows)
    v = _plain_values(s, s["v_pages"], 1, pages, rows)
    return _plain_masked(s, c, k, v, s["length"].long(), page >= 0)


def _plain_window(s, c):
    at = torch.arange(s["max_k"], device="cuda")
    row = (s["begin"].long()[:, None] + at).clamp(max=s["k"].shape[0] - 1)
    held = (s["end"] - s["begin"]).long()
    return _plain_masked(s, c, s["k"].float()[row], s["v"].float()[row], held, torch.ones_like(row, dtype=torch.bool))


def _plain_masked(s, c, k, v, held, live):
    """All sequences padded to the longest: scores, cap, mask, softmax, product."""
    hq, hk, d, tokens = c["heads"], c["kv"], c["dim"], s["q"].shape[0]
    grp = hq // hk
    off = s["offsets"].long()
    i = torch.arange(s["max_q"], device="cuda")
    j = torch.arange(s["max_k"], device="cuda")
    qi = (off[:-1, None] + i).clamp(max=tokens - 1)                      # [B, Q]
    q = s["q"].float()[qi].reshape(-1, s["max_q"], hk, grp, d).permute(0, 2, 3, 1, 4)       # [B, hk, grp, Q, d]
    x = torch.matmul(q, k.permute(0, 2, 3, 1)[:, :, None]) * (1 / math.sqrt(d))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    place = (s["start"].long()[:, None] + i)[:, :, None]                 # [B, Q, 1]
    see = j <= place
    if c["window"]:
        see = see & ((j > place - c["window"]) | (j < c["sinks"]))
    see = see & (live & (j < held[:, None]))[:, None]
    x = torch.where(see[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)[:, :, None]) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    at = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(off[1:].contiguous(), at, right=True)
    pick = seq * s["max_q"] + at - off[seq]
    o = o.permute(0, 3, 1, 2, 4).reshape(-1, hq, d)[pick]
    lse = lse[..., 0].permute(0, 3, 1, 2).reshape(-1, hq)[pick]
    return [o.to(s["q"].dtype), lse]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "pages":
        return None                                      # whole numbers, and copies
    s = prepare(case, seed)
    return _exact_write(s, case) if case["op"] == "write" else _exact_attention(s, case)


def _round8(x):
    """To the nearest 8-bit number of 4 exponent and 3 fraction bits, ties to the even one."""
    size = x.abs().clamp(min=2.0 ** -6)
    unit = torch.exp2(torch.floor(torch.log2(size)) - 3)
    unit = torch.where(size >= unit * 16, unit * 2, unit)
    unit = torch.where(size < unit * 8, unit / 2, unit)
    return torch.round(x / unit) * unit


def _exact_write(s, c):
    """Sequence by sequence, block by block."""
    new, held = _write_spans(c)
    kv, d, pr = c["kv"], c["dim"], c["page"]
    table, off = s["table"].tolist(), s["offsets"].tolist()
    if sum(-(-n // BLOCK) + 1 for n in new) > 6000:
        return None
    out = []
    scales = s["scales"].double()
    for which, x, pool in ((0, s["k"], s["k_pages"]), (1, s["v"], s["v_pages"])):
        val = pool.view(torch.float8_e4m3fn).double()
        for q, (n, h) in enumerate(zip(new, held)):
            for b in range(h // BLOCK, -(-(h + n) // BLOCK) if n else 0):
                lo, hi = max(h, b * BLOCK), min(h + n, (b + 1) * BLOCK)
                page, row = table[q][b * BLOCK // pr], b * BLOCK % pr
                y = x[off[q] + lo - h:off[q] + hi - h].double().transpose(0, 1)              # [kv, rows, d]
                top = y.abs().amax((1, 2))
                e = torch.ceil(torch.log2(top / 448))                    # a logarithm next to a whole number may miss it
                e = torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e)
                e = torch.where(448 * torch.exp2(e) < top, e + 1, e).clamp(E_MIN, E_MAX)
                if lo > b * BLOCK:
                    was = scales[page, :, row // BLOCK, which]
                    e = torch.maximum(e, was)
                    seen = val[page, :, row:row + lo - b * BLOCK]
                    val[page, :, row:row + lo - b * BLOCK] = _round8(seen * torch.exp2(was - e)[:, None, None])
                scales[page, :, row // BLOCK, which] = e
                val[page, :, row + lo - b * BLOCK:row + hi - b * BLOCK] = _round8(y * torch.exp2(-e)[:, None, None])
        out.append(val)
    return out + [None]


def _exact_attention(s, c):
    pairs, _ = _visible(c)
    if pairs * c["heads"] * c["dim"] > 1 << 40:
        return None
    n, held = _spans(c)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    at = 0
    for b, (m, h) in enumerate(zip(n, held)):
        if c["op"] == "attend":
            row = torch.arange(h, device="cuda")
            page, gone = s["table"][b, row // c["page"]].long(), s["table"][b, row // c["page"]] < 0
        for a in range(c["kv"]):
            if c["op"] == "attend":
                part = [p[page, a, row % c["page"]].view(torch.float8_e4m3fn).double()
                        * torch.exp2(s["scales"][page, a, row % c["page"] // BLOCK, w].double())[:, None]
                        for w, p in enumerate((s["k_pages"], s["v_pages"]))]
                kk, vv = part[0], part[1].masked_fill(gone[:, None], 0.0)
            else:
                lo = int(s["begin"][b])
                kk, vv = s["k"][lo:lo + h, a].double(), s["v"][lo:lo + h, a].double()
                gone = torch.zeros(h, dtype=torch.bool, device="cuda")
            for head in range(a * (c["heads"] // c["kv"]), (a + 1) * (c["heads"] // c["kv"])):
                for lo in range(0, m, 2048):
                    hi = min(m, lo + 2048)
                    x = s["q"][at + lo:at + hi, head].double() @ kk.T / math.sqrt(c["dim"])
                    if c["cap"]:
                        x = torch.tanh(x / c["cap"]) * c["cap"]
                    r = torch.arange(lo, hi, device="cuda")[:, None] + (h - m)
                    y = torch.arange(h, device="cuda")[None]
                    x.masked_fill_(y > r, -math.inf)
                    if c["window"]:
                        x.masked_fill_((r - y >= c["window"]) & (y >= c["sinks"]), -math.inf)
                    x.masked_fill_(gone[None], -math.inf)
                    t = torch.logsumexp(x, 1)
                    out[at + lo:at + hi, head] = torch.exp(x - t[:, None]).nan_to_num(0.0) @ vv
                    lse[at + lo:at + hi, head] = t
        at += m
    return [out, lse]
