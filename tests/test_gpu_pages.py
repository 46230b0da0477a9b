"""Paged token memory on the GPU against plain loops and the float64 form.

Tables, counts, copies and rounded numbers have to be equal.  Attention, with u the
output type's unit roundoff (2^-11 fp16, 2^-8 bf16) and A = sum_j p_j |v_j|: the
result's rounding costs u A, probabilities and widened values in 16 bits (many rows)
2 u A at most, a score error d costs 2 d A, float32 sums 2^-20 A.  d: float32 sums of
head_dim products (2^-23 of the largest sum of magnitudes times sqrt(head_dim)), tanh
to 4e-7 of the cap, the exponential to 2^-21; queries of bf16 scaled to fp16 lose
2^-39 of a row's largest, below the float32 sums' error.
"""
import math
import random

import numpy as np
import pytest

from tests import gpu_util as U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -133}
E_MIN, E_MAX = -120, 120


@pytest.fixture(scope="module")
def R():
    return U.load()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def full(n, v=-7):
    return torch.full(n if isinstance(n, tuple) else (n,), v, dtype=torch.int32, device="cuda")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ptr(t):
    return None if t is None or not t.numel() else t.data_ptr()


# ---------------------------------------------------------------------------
# fork, extend, compact
# ---------------------------------------------------------------------------

def fork_loop(parent, keep, window, sinks, length, table, per, pr, pages):
    out, rows, refs = [], [], [0] * pages
    for s, p in enumerate(parent):
        n = 0
        if 0 <= p < len(length):
            n = max(0, min(length[p], per * pr, keep[s] if keep else 1 << 30))
        row = []
        for i in range(per):
            e = table[p][i] if i * pr < n else -1
            if window and all(x >= sinks and x + window <= n for x in (i * pr, i * pr + pr - 1)):
                e = -1
            e = e if 0 <= e < pages else -1
            if e >= 0:
                refs[e] += 1
            row.append(e)
        out.append(n)
        rows.append(row)
    return out, rows, refs


@pytest.mark.parametrize("n,n_from,per,pr,pages", [(1, 1, 1, 32, 1), (7, 5, 9, 64, 50), (40, 60, 33, 32, 700),
                                                    (2000, 300, 11, 128, 3000), (3, 2, 4000, 32, 9000), (5, 0, 4, 64, 8)])
def test_fork_matches_the_loop(R, n, n_from, per, pr, pages):
    rng = random.Random(n * 31 + pages)
    for window, sinks in ((0, 0), (1, 0), (pr + 5, 3), (3 * pr, pr + 1)):
        length = [rng.choice([0, pr, per * pr, per * pr + 5, -3, rng.randint(0, per * pr)]) for _ in range(n_from)]
        table = [[rng.choice([rng.randrange(pages), rng.randrange(pages), -1, pages, -5]) for _ in range(per)]
                 for _ in range(n_from)]
        parent = [rng.choice([rng.randrange(-1, n_from + 1), 0]) for _ in range(n)]
        for keep in (None, [rng.randint(-2, per * pr + 9) for _ in range(n)]):
            want = fork_loop(parent, keep, window, sinks, length, table, per, pr, pages)
            cfg = R.page_config(1, 16, pr, pages, n, per)
            lo, to, refs = full(n), full((n, per)), full(pages)
            src_l, src_t = i32(length), i32(table).reshape(-1)
            par, kp = i32(parent), None if keep is None else i32(keep)
            R.check(R.rtcc_pages_fork(cfg, n_from, ptr(par), ptr(kp), window, sinks, ptr(src_l), ptr(src_t), ptr(lo), ptr(to),
                                      ptr(refs)))
            assert (lo.tolist(), to.tolist(), refs.tolist()) == want


@pytest.mark.parametrize("pr,window,sinks,back", [(32, 50, 4, 40), (64, 64, 0, 9), (128, 700, 130, 300)])
def test_fork_window_covers_what_is_taken_back(R, pr, window, sinks, back):
    """Forks with the attention's window and the tokens that may be taken back: after any number of
    steps a history shortened by up to that many still has every page that its tokens see.  With
    the attention's window alone some are gone."""
    rng = random.Random(pr)
    per, pages = 40, 200
    lost = 0
    for wide in (window + back, window):
        table, length = [list(range(per))], [0]
        for step in range(60):
            grown = min(per * pr, length[0] + rng.randint(1, back))
            row = [table[0][i] if i * pr < length[0] else i for i in range(per)]         # new pages for new places
            cfg = R.page_config(1, 16, pr, pages, 2, per)
            lo, to, refs = full(2), full((2, per)), full(pages)
            src_l, src_t, par = i32([grown]), i32(row), i32([0, 0])
            kp = i32([grown, max(0, grown - rng.randint(0, back))])
            R.check(R.rtcc_pages_fork(cfg, 1, ptr(par), ptr(kp), wide, sinks, ptr(src_l), ptr(src_t), ptr(lo), ptr(to), ptr(refs)))
            (m, short), rows = lo.tolist(), to.tolist()
            sees = [j for j in range(short) if j < sinks or j > short - window]          # of the next token at place `short`
            missing = [j for j in sees if rows[1][j // pr] < 0]
            lost += len(missing)
            assert wide == window or not missing
            table, length = [rows[0]], [m]
        assert wide == window or lost == 0
    assert lost > 0


def extend_loop(new, length, table, refs, pr):
    per, table, begin, refs = len(table[0]), [list(r) for r in table], list(refs), list(refs)
    free = [p for p, c in enumerate(begin) if c == 0]
    out, src, dst, rows, short = [], [], [], [], 0
    for s, n in enumerate(new):
        held = min(max(length[s], 0), per * pr)
        end = min(per * pr, held + max(n, 0))
        stop, copied = end, (-1, -1, 0)
        first = -(-held // pr)
        if end > held and held % pr:
            i = held // pr
            page = table[s][i]
            there = 0 <= page < len(refs)
            if not there or begin[page] > 1:
                if free:
                    got = free.pop(0)
                    table[s][i] = got
                    refs[got] = 1
                    if there:
                        refs[page] -= 1
                        copied = (page, got, held % pr)
                else:
                    short += 1
                    stop = held
                    if not there:
                        table[s][i] = -1
        for i in range(first, max(first, -(-end // pr))):
            if free:
                table[s][i] = free.pop(0)
                refs[table[s][i]] = 1
            else:
                short += 1
                table[s][i] = -1
                stop = max(held, min(stop, i * pr))
        out.append(stop)
        src.append(copied[0])
        dst.append(copied[1])
        rows.append(copied[2])
    return table, refs, out, src, dst, rows, short


@pytest.mark.parametrize("n,per,pr,pages,most", [(1, 1, 32, 1, 40), (1, 50, 32, 200, 2000), (9, 5, 64, 30, 90),
                                                  (60, 12, 32, 400, 50), (300, 7, 128, 5000, 300), (3000, 3, 64, 9001, 70),
                                                  (3000, 3, 64, 4001, 70), (4, 3, 32, 0, 20)])
def test_extend_matches_the_loop(R, n, per, pr, pages, most):
    rng = random.Random(n * 77 + pages)
    for round_ in range(3):
        length = [rng.choice([0, pr, rng.randint(0, per * pr), per * pr]) for _ in range(n)]
        new = [rng.choice([0, 1, rng.randint(-1, most)]) for _ in range(n)]
        order = list(range(pages))
        rng.shuffle(order)
        table, refs = [], [0] * pages
        for s in range(n):
            if s and rng.random() < 0.4:                        # shares its pages with the one before
                length[s] = length[s - 1]
                row = list(table[-1])
            else:
                row = [order.pop() if i * pr < length[s] and len(order) > pages // 4 else -1 for i in range(per)]
            for p in row:
                if p >= 0:
                    refs[p] += 1
            table.append(row)
        want = extend_loop(new, length, table, refs, pr)
        cfg = R.page_config(1, 16, pr, pages, n, per)
        t, c, nw, ln = i32(table), i32(refs), i32(new), i32(length)
        out, src, dst, rows, short = full(n), full(n), full(n), full(n), full(1)
        ws = torch.full((R.rtcc_pages_workspace(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
        if round_ == 1:
            out = ln                                            # lengths in place
        R.check(R.rtcc_pages_extend(cfg, ptr(nw), ptr(ln), ptr(t), ptr(c), ptr(out), ptr(src), ptr(dst), ptr(rows),
                                    None if round_ == 2 else ptr(short), ptr(ws), ws.numel()))
        got = (t.tolist(), c.tolist(), out.tolist(), src.tolist(), dst.tolist(), rows.tolist())
        assert got == want[:6]
        assert round_ == 2 or short.tolist() == [want[6]]


def compact_loop(table, refs):
    live = [p for p, c in enumerate(refs) if c > 0]
    n = len(live)
    src = [p for p in live if p >= n]
    dst = [p for p in range(n) if refs[p] <= 0]
    to = {p: p for p in live if p < n}
    to.update(zip(src, dst))
    out = [0] * len(refs)
    for p, q in to.items():
        out[q] = refs[p]
    return [[to.get(p, -1) for p in row] for row in table], out, src, dst


@pytest.mark.parametrize("n,per,pages,share", [(1, 1, 1, 1.0), (3, 4, 20, 0.0), (3, 4, 20, 1.0), (9, 30, 777, 0.3),
                                                (500, 9, 5000, 0.6), (50, 900, 20000, 0.5), (300, 300, 9999, 0.05)])
def test_compact_matches_the_loop(R, n, per, pages, share):
    rng = random.Random(n + pages)
    refs = [rng.randint(1, 4) if rng.random() < share else 0 for _ in range(pages)]
    table = [[rng.choice([rng.randrange(pages), -1, pages + 3]) for _ in range(per)] for _ in range(n)]
    want = compact_loop(table, refs)
    cfg = R.page_config(1, 16, 32, pages, n, per)
    ws = torch.full((R.rtcc_pages_workspace(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
    for in_place in (False, True):
        t, c = i32(table), i32(refs)
        to, ro, src, dst, count = t if in_place else full((n, per)), full(pages), full(pages), full(pages), full(1)
        R.check(R.rtcc_pages_compact(cfg, ptr(t), ptr(c), ptr(to), ptr(ro), ptr(src), ptr(dst), ptr(count), ptr(ws), ws.numel()))
        moves = count.item()
        assert moves == len(want[2])
        assert (to.tolist(), ro.tolist()) == want[:2]
        assert src.tolist() == want[2] + [-1] * (pages - moves) and dst.tolist() == want[3] + [-1] * (pages - moves)


def test_empty_tables(R):
    cfg = R.page_config(1, 16, 32, 40, 0, 5)
    refs, ws = full(40), torch.zeros(1024, dtype=torch.uint8, device="cuda")
    R.check(R.rtcc_pages_fork(cfg, 0, None, None, 0, 0, None, None, None, None, ptr(refs)))
    assert (refs == 0).all()
    short = full(1)
    R.check(R.rtcc_pages_extend(cfg, None, None, None, ptr(refs), None, None, None, None, ptr(short), ptr(ws), 1024))
    assert short.item() == 0 and (refs == 0).all()
    ro, src, dst, count = full(40), full(40), full(40), full(1)
    R.check(R.rtcc_pages_compact(cfg, None, ptr(refs), None, ptr(ro), ptr(src), ptr(dst), ptr(count), ptr(ws), 1024))
    assert count.item() == 0 and (ro == 0).all() and (src == -1).all()


# ---------------------------------------------------------------------------
# copy
# ---------------------------------------------------------------------------

def pool(pages, kv, pr, dim, g, page_pad=0, scale_pad=0):
    """Random codes and exponents, pages further apart by the pads."""
    n = kv * pr * dim
    k = torch.randint(0, 256, (pages, n + page_pad), generator=g, device="cuda", dtype=torch.uint8)
    v = torch.randint(0, 256, (pages, n + page_pad), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.randint(-9, 10, (pages, kv * (pr // 16) * 2 + scale_pad), generator=g, device="cuda", dtype=torch.int8)
    return k, v, s


@pytest.mark.parametrize("kv,pr,dim,pad", [(1, 32, 16, 0), (3, 64, 80, 16), (8, 128, 128, 0), (5, 32, 48, 4096)])
@pytest.mark.parametrize("partly", [False, True])
def test_copy_matches_the_loop(R, kv, pr, dim, pad, partly):
    g = gen(kv * pr)
    rng = random.Random(dim)
    a, b = pool(23, kv, pr, dim, g, pad, pad // 4), pool(40, kv, pr, dim, g, pad, pad // 4)
    n = 30
    dst = rng.sample(range(40), n)
    src = [rng.randrange(23) for _ in range(n)]
    for i, bad in ((3, -1), (9, 23), (17, -(2 ** 31))):
        src[i] = bad
    dst[11], dst[12] = -1, 40
    rows = [rng.choice([0, 1, 15, 16, 17, pr, pr + 9, -4]) for _ in range(n)] if partly else None
    want = [t.clone() for t in b]
    count = 27
    for i in range(count):
        if 0 <= src[i] < 23 and 0 <= dst[i] < 40:
            r = pr if rows is None else min(max(rows[i], 0), pr)
            m = kv * pr * dim
            for w in (0, 1):
                want[w][dst[i], :m].view(kv, pr, dim)[:, :r] = a[w][src[i], :m].view(kv, pr, dim)[:, :r]
            e = kv * (pr // 16) * 2
            want[2][dst[i], :e].view(kv, -1, 2)[:, :-(-r // 16)] = a[2][src[i], :e].view(kv, -1, 2)[:, :-(-r // 16)]
    cfg = R.page_config(kv, dim, pr, 23, 0, 0, page_bytes=a[0].stride(0), scale_bytes=a[2].stride(0))
    sd, dd, rd, cd = i32(src), i32(dst), None if rows is None else i32(rows), i32([count])
    R.check(R.rtcc_pages_copy(cfg, n, ptr(cd), ptr(sd), ptr(dd), ptr(rd), *[ptr(t) for t in a], 40, *[ptr(t) for t in b]))
    torch.cuda.synchronize()
    for x, y in zip(b, want):
        assert torch.equal(x, y)


def test_copy_past_32_bits(R):
    # pages 512 MB apart: the last one lies past 2^32 bytes
    step = 1 << 29
    big = torch.zeros(9 * step + 4096, dtype=torch.uint8, device="cuda")
    s = torch.zeros(10, 4, dtype=torch.int8, device="cuda")
    big[9 * step:9 * step + 512] = torch.arange(512, device="cuda").to(torch.uint8)
    s[9] = 5
    cfg = R.page_config(1, 16, 32, 10, 0, 0, page_bytes=step, scale_bytes=4)
    src, dst = i32([9]), i32([1])
    v = big[1024:]
    v[9 * step:9 * step + 512] = 3
    R.check(R.rtcc_pages_copy(cfg, 1, None, ptr(src), ptr(dst), None, big.data_ptr(), v.data_ptr(), ptr(s), 10, big.data_ptr(),
                              v.data_ptr(), ptr(s)))
    torch.cuda.synchronize()
    assert torch.equal(big[step:step + 512], big[9 * step:9 * step + 512]) and (v[step:step + 512] == 3).all()
    assert (s[1] == 5).all() and (s[2] == 0).all()


# ---------------------------------------------------------------------------
# write
# ---------------------------------------------------------------------------

GRID = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()     # 0 .. 448


def round8(x):
    """To the nearest e4m3 number by looking through all of them, ties to the even code; as codes."""
    mag = np.abs(x)
    hi = np.clip(np.searchsorted(GRID, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = (GRID[hi] - mag < mag - GRID[lo]) | ((GRID[hi] - mag == mag - GRID[lo]) & (hi % 2 == 0))
    code = np.where(mag >= GRID[126], 126, np.where(up, hi, lo)).astype(np.uint8)
    code = code | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isnan(x), 0x7F, code)


def need(top):
    e = E_MIN
    if top > 0:
        m, x = math.frexp(top)
        e = min(max(x - 9 + (m > 0.875), E_MIN), E_MAX)
    return e


def write_loop(x, new, held, limit, table, codes, exps, which, pr):
    """Loops over sequences, blocks and heads on numpy arrays, in place."""
    at = 0
    for s, n in enumerate(new):
        end = min(held[s] + n, limit[s], len(table[s]) * pr)
        for b in range(held[s] // 16, -(-end // 16)):
            lo, hi = max(held[s], b * 16), min(end, b * 16 + 16)
            if hi <= lo:
                continue
            page, row = table[s][b * 16 // pr], b * 16 % pr
            if not 0 <= page < codes.shape[0]:
                continue
            for h in range(codes.shape[1]):
                y = x[at + lo - held[s]:at + hi - held[s], h]
                fine = np.isfinite(y)
                e = need(np.abs(y[fine]).max() if fine.any() else 0.0)
                old = exps[page, h, row // 16, which]
                if lo > b * 16:
                    e = max(e, int(old))
                    if e > old:
                        z = codes[page, h, row:row + lo - b * 16]
                        v = np.where(z & 0x7F == 0x7F, np.nan, GRID[np.minimum(z & 0x7F, 126)] * np.where(z >> 7, -1.0, 1.0))
                        codes[page, h, row:row + lo - b * 16] = np.where(np.isnan(v), z | 0x7F, round8(v * 2.0 ** (int(old) - e)))
                exps[page, h, row // 16, which] = e
                c = round8(np.where(fine, y, np.nan) * 2.0 ** -e)
                codes[page, h, row + lo - b * 16:row + hi - b * 16] = c
        at += n


def same_codes(a, b):
    """Equal, where all NaN codes count as one."""
    a, b = a.astype(np.uint8), b.astype(np.uint8)
    return bool(((a == b) | ((a & 0x7F == 0x7F) & (b & 0x7F == 0x7F))).all())


@pytest.mark.parametrize("dim,kv,pr,dtype", [(16, 1, 32, "fp16"), (32, 3, 64, "bf16"), (48, 2, 32, "fp16"), (64, 2, 64, "bf16"),
                                              (80, 3, 128, "fp16"), (96, 1, 64, "bf16"), (112, 2, 32, "bf16"),
                                              (128, 5, 128, "fp16"), (128, 2, 64, "bf16")])
def test_write_matches_the_loop(R, dim, kv, pr, dtype):
    g = gen(dim + kv)
    new = [1, 16, 17, 40, 0, 3, 1, 130, 15, 5]
    held = [0, 0, 9, 16, 20, 31, 47, 5, 1, 100]
    limit = [1 << 30] * 9 + [102]                              # the last one has pages for two of its five
    per = 6
    n_pages = 60
    order = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    table = [[order.pop() if i * pr < held[s] + new[s] else -1 for i in range(per)] for s in range(len(new))]
    table[3][0] = -1                                           # a page that is missing
    limit[1] = 16
    n = sum(new)
    x = torch.randn(2, n, kv, dim + 8, generator=g, device="cuda") * torch.exp2(
        torch.randint(-12, 8, (2, n, kv, 1), generator=g, device="cuda").float())
    x[:, ::7] *= 0.0
    x[0, 3, 0, 1], x[0, 20, 0, 2], x[1, 5, 0, 0] = float("inf"), float("nan"), float("-inf")
    x = x.to(DT[dtype])
    k, v = x[0, ..., :dim], x[1, ..., :dim]
    kp, vp, sc = pool(n_pages, kv, pr, dim, g, 32, 4)
    m, e = kv * pr * dim, kv * (pr // 16) * 2
    want = [t[:, :m].cpu().numpy().reshape(n_pages, kv, pr, dim).copy() for t in (kp, vp)]
    exps = sc[:, :e].cpu().numpy().reshape(n_pages, kv, pr // 16, 2).copy()
    for which, t in ((0, k), (1, v)):
        write_loop(t.double().cpu().numpy(), new, held, limit, table, want[which], exps, which, pr)
    cfg = R.page_config(kv, dim, pr, n_pages, len(new), per, page_bytes=kp.stride(0), scale_bytes=sc.stride(0))
    off = i32(np.concatenate([[0], np.cumsum(new)]))
    hd, ln, tb = i32(held), i32(limit), i32(table)
    first = [t.clone() for t in (kp, vp, sc)]
    for most in (1, max(new), 10 ** 6):
        for t, f in zip((kp, vp, sc), first):
            t.copy_(f)
        tok = R.write_config(R.BF16 if dtype == "bf16" else R.FP16, n, most, k.stride()[:2], v.stride()[:2])
        R.check(R.rtcc_pages_write(cfg, tok, ptr(k), ptr(v), ptr(off), ptr(hd), ptr(ln), ptr(tb), ptr(kp), ptr(vp), ptr(sc)))
        torch.cuda.synchronize()
        for got, w in zip((kp, vp), want):
            assert same_codes(got[:, :m].cpu().numpy().reshape(w.shape), w)
        assert (sc[:, :e].cpu().numpy().reshape(exps.shape) == exps).all()
        assert torch.equal(kp[:, m:], first[0][:, m:]) and torch.equal(sc[:, e:], first[2][:, e:])


def test_write_every_number_and_extremes(R):
    """All finite 16-bit numbers of each sign, one block each; the largest and smallest of a type."""
    for dtype in ("fp16", "bf16"):
        codes = torch.arange(0, 1 << 16, device="cuda").to(torch.int32).to(torch.int16).view(DT[dtype])
        n = codes.numel() // 16
        k = codes.view(n, 1, 16).contiguous()                   # 16 neighbouring numbers of one token, 16 tokens to a block
        cfg = R.page_config(1, 16, 128, n // 128, 1, n // 128)
        kp, vp = (torch.zeros(n // 128, 1, 128, 16, dtype=torch.uint8, device="cuda") for _ in range(2))
        sc = torch.zeros(n // 128, 1, 8, 2, dtype=torch.int8, device="cuda")
        table, off, held = i32(list(range(n // 128))), i32([0, n]), i32([0])
        tok = R.write_config(R.BF16 if dtype == "bf16" else R.FP16, n, n, (16, 16), (16, 16))
        R.check(R.rtcc_pages_write(cfg, tok, ptr(k), ptr(k), ptr(off), ptr(held), None, ptr(table), ptr(kp), ptr(vp), ptr(sc)))
        torch.cuda.synchronize()
        x = k.double().cpu().numpy().reshape(-1, 256)           # a block: 16 tokens of 16
        fine = np.isfinite(x)
        e = np.array([need(np.abs(r[f]).max() if f.any() else 0.0) for r, f in zip(x, fine)])
        assert (sc[..., 0].cpu().numpy().reshape(-1) == e).all() and (sc[..., 1] == sc[..., 0]).all()
        want = round8(np.where(fine, x, np.nan) * 2.0 ** -e[:, None].astype(np.float64))
        assert same_codes(kp.cpu().numpy().reshape(want.shape), want) and torch.equal(kp, vp)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

class Case:
    """Random sequences on shuffled pages; whatever no token sees holds NaN codes and wild exponents."""

    def __init__(self, n, m, heads=2, kv=1, dim=64, pr=64, dtype="fp16", causal=True, window=0, sinks=0, prefix=None, cap=0.0,
                 start=None, missing=(), spread=1.0, seed=0, lse=True, per=None, pad=0):
        g = gen(seed + 500)
        self.n, self.m, self.heads, self.kv, self.dim, self.pr, self.dtype = list(n), list(m), heads, kv, dim, pr, dtype
        self.causal, self.window, self.sinks, self.prefix, self.cap = causal, window, sinks, prefix, cap
        self.start = [b - a for a, b in zip(n, m)] if start is None else list(start)
        self.given, self.scale, self.tokens = start is not None, 1 / math.sqrt(dim), sum(n)
        self.per = per or max(1, max(-(-x // pr) for x in m))
        self.pages = sum(-(-x // pr) for x in m) + 3
        order = torch.randperm(self.pages, generator=g, device="cuda").tolist()
        self.table = [[order.pop() if i * pr < m[s] else -1 for i in range(self.per)] for s in range(len(m))]
        for s, i in missing:
            self.table[s][i] = -1
        self.q = (spread * torch.randn(self.tokens, heads, dim + 8, generator=g, device="cuda")).to(DT[dtype])[..., :dim]
        nb = pr // 16
        size = kv * pr * dim
        self.k, self.v, self.s = pool(self.pages, kv, pr, dim, g, pad, pad // 4)
        # numbers up to about 3 with exponents of blocks from -8 to -5
        for which, t in ((0, self.k), (1, self.v)):
            x = torch.randn(self.pages, kv, nb, 16, dim, generator=g, device="cuda")
            e = torch.randint(-8, -4, (self.pages, kv, nb), generator=g, device="cuda")
            c = torch.ldexp(x, -e[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            t[:, :size] = c.view(self.pages, size)
            self.s[:, :kv * nb * 2].view(self.pages, kv, nb, 2)[..., which] = e.to(torch.int8)
        seen = torch.zeros(self.pages, pr, dtype=torch.bool)
        for s in range(len(m)):
            see = self.visible(s).any(0)
            for j in np.nonzero(see)[0]:
                seen[self.table[s][j // pr], j % pr] = True
        seen = seen.cuda()
        hide = ~seen[:, None, :, None].expand(self.pages, kv, pr, dim)
        for t in (self.k, self.v):
            x = t[:, :size].view(self.pages, kv, pr, dim)
            x[hide] = 0x7F
        none = ~seen.view(self.pages, nb, 16).any(-1)[:, None, :, None].expand(self.pages, kv, nb, 2)
        self.s[:, :kv * nb * 2].view(self.pages, kv, nb, 2)[none] = 127
        self.out = torch.full((self.tokens, heads, dim), 7.0, device="cuda", dtype=DT[dtype])
        self.lse = torch.full((self.tokens, heads), 7.0, device="cuda") if lse else None

    def visible(self, s):
        n, m = self.n[s], self.m[s]
        p, j = np.arange(n)[:, None] + self.start[s], np.arange(m)[None]
        see = np.ones((n, m), dtype=bool)
        if self.causal:
            see = j <= p
            if self.window:
                see = see & ((j > p - self.window) | (j < self.sinks))
            if self.prefix is not None:
                see = see | (j < self.prefix[s])
        live = np.array([self.table[s][x // self.pr] >= 0 for x in range(m)], dtype=bool)
        return see & live[None]

    def values(self, s, which, h):
        t = (self.k, self.v)[which][:, :self.kv * self.pr * self.dim].view(self.pages, self.kv, self.pr, self.dim)
        e = self.s[:, :self.kv * (self.pr // 16) * 2].view(self.pages, self.kv, self.pr // 16, 2)
        j = torch.arange(self.m[s], device="cuda")
        page = torch.tensor(self.table[s], device="cuda")[j // self.pr].clamp(min=0)
        x = t[page, h, j % self.pr].view(torch.float8_e4m3fn).double()
        return x * torch.exp2(e[page, h, j % self.pr // 16, which].double())[:, None]

    def run(self, R, workspace=64 << 20, max_q=None, max_k=None, stream=0):
        self.off_d, self.l_d = i32(np.concatenate([[0], np.cumsum(self.n)])), i32(self.m)
        self.t_d, self.p_d = i32(self.table), None if self.prefix is None else i32(self.prefix)
        self.s_d = i32(self.start) if self.given else None
        self.ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        cfg = R.page_config(self.kv, self.dim, self.pr, self.pages, len(self.n), self.per, page_bytes=self.k.stride(0),
                            scale_bytes=self.s.stride(0))
        rows = R.page_attn_config(self.heads, R.BF16 if self.dtype == "bf16" else R.FP16, self.tokens, self.q.stride()[:2],
                                  self.out.stride()[:2], max(self.n + [0]) if max_q is None else max_q,
                                  max(self.m + [0]) if max_k is None else max_k, causal=self.causal, window=self.window,
                                  sinks=self.sinks, scale=self.scale, cap=self.cap)
        self.args = [cfg, rows, ptr(self.q), ptr(self.off_d), ptr(self.s_d), ptr(self.l_d), ptr(self.p_d), ptr(self.t_d),
                     ptr(self.k), ptr(self.v), ptr(self.s), ptr(self.out), ptr(self.lse),
                     self.ws.data_ptr() if workspace else None, workspace]
        R.check(R.rtcc_pages_attention(*self.args, stream))
        return self

    def check(self):
        torch.cuda.synchronize()
        u, at = ROUND[self.dtype], 0
        for s, (n, m) in enumerate(zip(self.n, self.m)):
            see = torch.tensor(self.visible(s), device="cuda").reshape(n, m)
            for h in range(self.heads):
                kh = h // (self.heads // self.kv)
                kk = torch.where(see.any(0)[:, None], self.values(s, 0, kh), 0.0)
                vv = torch.where(see.any(0)[:, None], self.values(s, 1, kh), 0.0)
                qq = self.q[at:at + n, h].double()
                x = self.scale * (qq @ kk.T)
                size = self.scale * float((qq.abs() @ kk.abs().T).max()) if n and m else 0.0
                if self.cap:
                    x = self.cap * torch.tanh(x / self.cap)
                x = torch.where(see, x, -math.inf)
                lse = torch.logsumexp(x, 1) if m else torch.full((n,), -math.inf, device="cuda", dtype=torch.float64)
                p = torch.where(see, torch.exp(x - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
                want, A = p @ vv, p @ vv.abs()
                d = 2.0 ** -23 * math.sqrt(self.dim) * size + 4e-7 * self.cap + 2.0 ** -21
                err = (self.out[at:at + n, h].double() - want).abs()
                lim = (2 * u + 2 * d + 2.0 ** -20) * A + TINY[self.dtype]
                assert bool((err <= lim).all()), (s, h, float((err / lim).max()))
                if self.lse is not None:
                    gl = self.lse[at:at + n, h].double()
                    none = torch.isinf(lse)
                    assert bool((gl[none] == -math.inf).all())
                    e = (gl - lse).abs()[~none]
                    assert bool((e <= d + 2.0 ** -20 * (1 + lse[~none].abs())).all()), float(e.max())
            at += n
        return self


LENGTHS = [([1], [1]), ([1], [0]), ([1], [63]), ([1], [129]), ([2], [5000]), ([16], [257]), ([17], [1000]), ([127], [127]),
           ([128], [128]), ([129], [385]), ([257], [1023]), ([300], [20000]), ([1, 1, 1, 1], [1, 0, 777, 4096]),
           ([0, 3, 0, 40], [10, 3, 0, 200]), ([5, 64, 200, 1], [0, 64, 333, 1])]


@pytest.mark.parametrize("n,m", LENGTHS)
@pytest.mark.parametrize("dim,heads,kv,pr,dtype", [(64, 2, 2, 32, "fp16"), (128, 4, 1, 64, "bf16")])
@pytest.mark.parametrize("causal", [False, True])
def test_pages_lengths(R, n, m, dim, heads, kv, pr, dtype, causal):
    Case(n, m, heads, kv, dim, pr, dtype, causal=causal).run(R).check()


@pytest.mark.parametrize("n,m", [(1, 1500), (9, 700), (150, 700)])
@pytest.mark.parametrize("dim", [16, 32, 48, 80, 96, 112, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_pages_head_sizes(R, n, m, dim, dtype):
    Case([n, n], [m, m - 35], 3, 1, dim, 128, dtype, pad=48).run(R).check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (12, 4), (16, 1), (40, 2), (130, 1), (129, 1)])
@pytest.mark.parametrize("n,m", [(1, 300), (3, 200), (60, 130)])
def test_pages_head_groups(R, heads, kv, n, m):
    Case([n], [m], heads, kv, 64, 32).run(R).check()


@pytest.mark.parametrize("n,m,window,sinks", [
    ([1], [500], 1, 0), ([1], [5000], 700, 16), ([1], [5000], 9000, 4), ([3], [1000], 50, 70), ([40], [3000], 333, 130),
    ([100], [100], 1, 0), ([130], [130], 7, 200), ([200], [5000], 640, 64), ([300], [300], 64, 0), ([700], [700], 100, 10),
    ([257], [10000], 2000, 65), ([1, 1, 1, 1], [1, 0, 777, 4096], 300, 5), ([300, 129], [290, 5000], 128, 128)])
@pytest.mark.parametrize("dim,heads,kv,pr,dtype", [(64, 2, 2, 128, "bf16"), (128, 4, 1, 32, "fp16")])
def test_pages_windows(R, n, m, window, sinks, dim, heads, kv, pr, dtype):
    Case(n, m, heads, kv, dim, pr, dtype, window=window, sinks=sinks).run(R).check()


@pytest.mark.parametrize("n,m", [(1, 1000), (20, 1000), (150, 1300), (400, 400)])
def test_pages_prefix_starts_and_caps(R, n, m):
    Case([n, n], [m, m], 4, 2, 64, 64, prefix=[100, 333], window=64, sinks=5).run(R).check()
    Case([n, n], [m, m], 4, 2, 64, 64, prefix=[0, m], cap=20.0, spread=3.0).run(R).check()
    Case([n, n], [m, m], 2, 1, 128, 32, "bf16", start=[m - n // 2, 100], cap=500.0).run(R).check()
    Case([n], [m], 2, 1, 64, 64, start=[m - n // 2], window=90, sinks=4).run(R).check()


@pytest.mark.parametrize("n", [1, 20, 200])
def test_pages_missing(R, n):
    """Entries that name no page hide their keys, at the ends, in the middle, all of them."""
    for pr, missing in ((32, ((0, 0), (0, 3), (0, 4), (1, 5))), (64, ((0, 2), (0, 14), (1, 0))),
                        (128, tuple((0, i) for i in range(8)))):
        Case([n, n], [1000, 300], 2, 1, 64, pr, missing=missing).run(R).check()
        Case([n, n], [1000, 300], 2, 1, 64, pr, missing=missing, window=300, sinks=40).run(R).check()


# sizes that the tensor-core kernel takes: more than 128 rows of a key head, and more than
# 300,000 pairs of a block of 16 of them and a key
@pytest.mark.parametrize("n,m", [([1500], [1500]), ([700, 900], [2700, 900]), ([1300], [5000]), ([600, 1, 0, 65], [4096, 900, 10, 3000]),
                                 ([1025], [1020])])
@pytest.mark.parametrize("dim,heads,kv,pr,dtype", [(64, 4, 4, 32, "fp16"), (128, 4, 2, 64, "bf16"), (80, 6, 3, 128, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 10), (640, 64), (1, 0)])
def test_pages_large(R, n, m, dim, heads, kv, pr, dtype, window, sinks):
    Case(n, m, heads, kv, dim, pr, dtype, window=window, sinks=sinks, pad=16).run(R).check()


@pytest.mark.parametrize("dim", [16, 48, 96, 112])
def test_pages_large_heads_scores_and_starts(R, dim):
    Case([1200, 700], [1300, 2000], 4, 4, dim, 64, "bf16", cap=20.0, spread=3.0).run(R).check()
    Case([1200, 700], [1300, 2000], 4, 4, dim, 64, "fp16", cap=500.0, window=300, sinks=7).run(R).check()
    Case([1200, 700], [1300, 2000], 4, 4, dim, 32, "fp16", prefix=[100, 1999], window=64, sinks=5).run(R).check()
    Case([1200, 700], [1300, 2000], 8, 4, dim, 128, "fp16", start=[700, 1500]).run(R).check()
    Case([1200], [1300], 8, 4, dim, 128, "fp16", causal=False).run(R).check()


def test_pages_large_missing(R):
    """Entries that name no page hide their keys: halves of steps, whole steps, the sequence's ends, all of it."""
    for pr, missing in ((32, ((0, 0), (0, 3), (0, 8), (0, 9), (0, 46), (1, 5))), (64, ((0, 2), (0, 22), (1, 0))),
                        (128, tuple((0, i) for i in range(12)))):
        Case([1500, 600], [1500, 900], 4, 4, 64, pr, missing=missing).run(R).check()
        Case([1500, 600], [1500, 900], 4, 4, 64, pr, missing=missing, window=300, sinks=40).run(R).check()


@pytest.mark.parametrize("n,m,window", [(1, 60000, 0), (2, 9000, 8000), (40, 9000, 3000), (300, 9000, 0)])
def test_pages_split(R, n, m, window):
    """With and without room for parts or widened keys: the same result."""
    for workspace in (0, 200000, 3 << 20, 64 << 20):
        Case([n, 3], [m, 200], 2, 1, 64, 64, window=window, sinks=33 if window else 0).run(R, workspace=workspace).check()


@pytest.mark.parametrize("n", [3, 200, 1500])
def test_pages_limits_cut(R, n):
    """Tokens from max_q on and keys from max_k on are left out."""
    for max_q, max_k in ((n - 2, 1000), (n, 500), (1, 64), (0, 1000), (n, 0)):
        c = Case([n], [1000], 8, 8, 64, 64, causal=False).run(R, max_q=max_q, max_k=max_k)
        torch.cuda.synchronize()
        assert (c.out[max_q:] == 7).all()
        ref = Case([n], [1000], 8, 8, 64, 64, causal=False)
        ref.m = [max_k]
        ref.out, ref.lse = c.out[:max_q], c.lse[:max_q]
        ref.n = [max_q]
        ref.check()


class Limited(Case):
    """Tokens from most_q on and keys from most_k on are left out; what no token that is left sees holds NaN."""

    def __init__(self, n, m, most_q, most_k, **kw):
        self.most_q, self.most_k = most_q, most_k
        super().__init__(n, m, **kw)

    def visible(self, s):
        see = super().visible(s)
        see[self.most_q:] = False
        see[:, self.most_k:] = False
        return see

    def run(self, R, **kw):
        return super().run(R, max_q=self.most_q, max_k=self.most_k, **kw)

    def check(self):
        torch.cuda.synchronize()
        at = 0
        for n in self.n:
            out, lse = self.out[at + min(n, self.most_q):at + n], self.lse[at + min(n, self.most_q):at + n]
            assert bool((out == 7).all()) and bool((lse == 7).all())
            out.zero_()
            lse.fill_(-math.inf)
            at += n
        return super().check()


@pytest.mark.parametrize("n,m,most_q", [([9, 4], [300, 900], 3), ([200, 30], [700, 900], 60), ([3000, 20, 900], [4000, 700, 900], 1000),
                                         ([2500], [2500], 1400), ([1700, 1600], [300, 1500], 1500)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 10), (640, 64), (1, 0)])
@pytest.mark.parametrize("given", [False, True])
def test_pages_left_out_tokens_and_their_keys(R, n, m, most_q, window, sinks, given):
    """Causal: keys that only left-out tokens would see are not read, and may hold anything, those
    in the last step of what is read too."""
    start = [max(0, b - a) for a, b in zip(n, m)] if given else None
    Limited(n, m, most_q, max(m), heads=4, kv=4, dim=64, pr=64, window=window, sinks=sinks, start=start).run(R).check()
    if not given:
        Limited(n, m, most_q, max(m), heads=4, kv=2, dim=80, pr=32, dtype="bf16", window=window, sinks=sinks,
                prefix=[x // 3 for x in m]).run(R).check()


@pytest.mark.parametrize("n,m,most_k", [([1], [1000], 500), ([3, 40], [1000, 300], 400), ([200, 90], [700, 1500], 600),
                                         ([1500, 30], [3000, 900], 2000), ([1300], [1300], 1000)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 10), (640, 64)])
@pytest.mark.parametrize("given", [False, True])
def test_pages_left_out_keys_move_no_token(R, n, m, most_k, window, sinks, given):
    """Keys from max_k on are left out; the tokens stay where they were."""
    start = [b - a for a, b in zip(n, m)] if given else None
    Limited(n, m, max(n), most_k, heads=4, kv=4, dim=64, pr=64, window=window, sinks=sinks, start=start).run(R).check()
    Limited(n, m, max(n), most_k, heads=4, kv=2, dim=128, pr=32, dtype="bf16", window=window, sinks=sinks, start=start,
            prefix=[x // 4 for x in m]).run(R).check()


@pytest.mark.parametrize("n,m", [(1, 1000), (8, 1000), (200, 777), (1300, 1500)])
def test_pages_starts_behind_the_keys(R, n, m):
    for window, sinks in ((0, 0), (50, 7), (640, 64), (3000, 0)):
        for start in ([m, m + 30], [m + 100, m - n], [2 ** 31 - 1, m + window]):
            Case([n, n], [m, m], 4, 4, 64, 64, window=window, sinks=sinks, start=start).run(R).check()


def test_pages_exponents_far_apart(R):
    """Blocks from 2^-100 to 2^100: none overflows, none of the large ones is lost."""
    for n in (1, 40):
        c = Case([n], [400], 2, 1, 64, 64, "bf16", causal=False)
        e = torch.randint(-100, 101, (c.pages, 4), generator=gen(3), device="cuda").to(torch.int8)
        c.s.view(c.pages, 1, 4, 2)[:, 0, :, 1] = e
        c.run(R).check()


def test_pages_large_values_that_hardly_count(R):
    """A block of values up to 2^60 whose keys have scores 96 below the others': its share is
    2^-70 of the result, and the others keep their digits."""
    for n in (1, 40, 3000):
        c = Case([n], [400], 8, 4, 64, 64, "bf16", causal=False)
        c.q = torch.full_like(c.q, 4.0)
        page, row = c.table[0][2], 16
        c.k.view(c.pages, 4, 64, 64)[page, :, row:row + 16] = torch.tensor(-3.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
        s = c.s.view(c.pages, 4, 4, 2)
        s[page, :, row // 16, 0], s[page, :, row // 16, 1] = 0, 52
        s[..., 0].sub_((s[..., 0] != 0).to(torch.int8))        # the others' keys are small
        c.run(R).check()


def one_number(c, which, page, row, x):
    """All channels and heads of place `row` of a page: the e4m3 number x."""
    t = (c.k, c.v)[which][:, :c.kv * c.pr * c.dim].view(c.pages, c.kv, c.pr, c.dim)
    t[page, :, row] = torch.tensor(float(x)).to(torch.float8_e4m3fn).view(torch.uint8).item()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [1.3e7, 2e8, -2e8, 1e9, -1e9, 1e12, -1e30])
def test_pages_large_scores(R, dtype, size):
    """Scores beyond 2^24, where float32 has no fractions left: a token's only key, or the one
    whose score is a sixteenth of all scores above the next, is the result, whatever the sizes
    of the values.  One rounding of the result and one of the weight: 2 u |v|."""
    u = ROUND[dtype]
    for n, kv, window in ((1, 1, 0), (1, 1, 1), (40, 1, 0), (40, 1, 1), (1500, 4, 0), (1500, 4, 1)):
        c = Case([n], [1500], 4 * kv if n == 1 else kv, kv, 64, 64, dtype, causal=window > 0, window=window)
        c.s.view(c.pages, kv, 4, 2)[..., 0] = -3
        keys = torch.tensor([1.0 + i / 16 for i in range(4)] * 375)[torch.randperm(1500, generator=torch.Generator().manual_seed(1))]
        best = 777
        keys[best] = 2.0 if size > 0 else 0.8125
        for j in range(1500):
            one_number(c, 0, c.table[0][j // 64], j % 64, keys[j])
        c.q = torch.full_like(c.q, 1024.0)
        c.scale = size / (64 * 1024.0 * (0.25 if size > 0 else 0.8125 / 8))         # the winner's score is `size`
        c.run(R)
        torch.cuda.synchronize()
        for h in range(c.heads):
            v = c.values(0, 1, h // (c.heads // kv))
            want = v[1500 - n:] if window else v[best].expand(n, 64)
            assert bool(((c.out[:, h].double() - want).abs() <= 2 * u * want.abs() + TINY[dtype]).all()), (n, window)
            k = c.values(0, 0, h // (c.heads // kv))[:, 0]
            top = size * (k[1500 - n:] / k[best] if window else torch.ones_like(k[:n]))
            assert bool(((c.lse[:, h].double() - top).abs() <= 2.0 ** -20 * top.abs()).all()), (n, window)


@pytest.mark.parametrize("size", [1.3e7, -1e9])
def test_pages_large_scores_alike(R, size):
    """Few rows, all scores the same large number: the values' mean, though their exponents differ."""
    for n in (1, 40):
        c = Case([n], [700], 2, 1, 64, 64, causal=False)
        c.s.view(c.pages, 1, 4, 2)[..., 0] = -3
        c.s.view(c.pages, 1, 4, 2)[:, 0, :, 1] = torch.randint(-9, 3, (c.pages, 4), generator=gen(2), device="cuda").to(torch.int8)
        for j in range(700):
            one_number(c, 0, c.table[0][j // 64], j % 64, 1.0)
        c.q = torch.full_like(c.q, 1024.0)
        c.scale = size / (64 * 1024.0 / 8)
        c.run(R)
        torch.cuda.synchronize()
        v = c.values(0, 1, 0)
        want, A = v.mean(0), v.abs().mean(0)
        # one rounding of the result, one of the weights, float32 sums
        assert bool(((c.out.double() - want).abs() <= (2 * 2.0 ** -11 + 2.0 ** -20) * A + TINY["fp16"]).all())


def test_pages_wide_queries(R):
    """bf16 queries far outside fp16's range, scores of ordinary size."""
    for n in (1, 40):
        for shift in (60, -60):
            c = Case([n], [400], 2, 1, 64, 64, "bf16")
            c.q = c.q * 2.0 ** shift
            c.scale = c.scale * 2.0 ** -shift
            c.run(R).check()


def test_pages_non_finite_stays_in_its_rows(R):
    for n in (1, 30, 200):
        ref = Case([n, 5], [300, 300], 2, 2).run(R).check()
        c = Case([n, 5], [300, 300], 2, 2)
        c.q[0, 0, 3] = float("nan")
        c.run(R)
        torch.cuda.synchronize()
        assert torch.isnan(c.out[0, 0]).all() and torch.isnan(c.lse[0, 0])
        same = torch.ones(n + 5, 2, dtype=torch.bool, device="cuda")
        same[0, 0] = False
        assert torch.equal(c.out[same], ref.out[same]) and torch.equal(c.lse[same], ref.lse[same])


@pytest.mark.parametrize("window,sinks,cap", [(0, 0, 0.0), (300, 9, 0.0), (300, 9, 20.0), (1, 0, 0.0)])
def test_pages_large_non_finite_stays_in_its_rows(R, window, sinks, cap):
    """The kernel for many rows: queries with NaN or infinities make their own rows NaN, no other."""
    c = Case([1500, 40], [1500, 900], 4, 4, window=window, sinks=sinks, cap=cap)
    q = c.q.clone()
    bad = [(0, 0), (130, 1), (700, 3), (1499, 2), (1510, 0)]
    for i, (t, h) in enumerate(bad):
        c.q[t, h, 3 + i] = float("nan" if i % 2 == 0 else "inf")
        if i % 2:
            c.q[t, h, 9] = float("nan")
    c.run(R)
    torch.cuda.synchronize()
    ref = Case([1500, 40], [1500, 900], 4, 4, window=window, sinks=sinks, cap=cap).run(R).check()
    for t, h in bad:
        assert torch.isnan(c.out[t, h]).all() and torch.isnan(c.lse[t, h])
        c.out[t, h], c.lse[t, h] = ref.out[t, h], ref.lse[t, h]
    c.q.copy_(q)
    c.check()


class Narrow(Case):
    """Keys and values as fp16 has them: cut to its largest, rounded to multiples of its smallest."""

    def values(self, s, which, h):
        return super().values(s, which, h).clamp(-65504, 65504).half().double()


@pytest.mark.parametrize("up", [True, False])
def test_pages_fp16_queries_over_what_fp16_cannot_hold(R, up):
    """Pools of bf16 tokens and fp16 queries: few rows take the numbers as they are, many rows as
    fp16 has them."""
    for n, kv, kind in ((1, 1, Case), (40, 1, Case), (1500, 4, Narrow)):
        c = kind([n], [1500], kv, kv, 64, 64, causal=False)
        g = gen(4)
        if up:                                               # keys up to 448 * 2^13, queries to match
            c.s.view(c.pages, kv, 4, 2)[..., 0] = torch.randint(6, 14, (c.pages, kv, 4), generator=g, device="cuda").to(torch.int8)
            c.scale *= 2.0 ** -14
        else:                                                # keys around 2^-26, values around 2^-20
            e = torch.randint(-36, -30, (c.pages, kv, 4), generator=g, device="cuda").to(torch.int8)
            c.s.view(c.pages, kv, 4, 2)[..., 0], c.s.view(c.pages, kv, 4, 2)[..., 1] = e, e + 8
            c.scale *= 2.0 ** 24
        x, w = (torch.abs(Case.values(c, 0, which, 0)) for which in (0, 1))
        assert bool((x > 65504).any()) if up else bool((x < 2.0 ** -25).any()) and bool((w < 2.0 ** -14).any())
        c.run(R).check()


def test_pages_more_sequences_than_a_grid_is_high(R):
    """70,000 sequences, the first 69,997 of them empty."""
    c = Case([150, 3, 40], [64, 60, 33], 2, 1, 16, 32).run(R).check()
    more = 69997
    off, length = i32([0] * more + [0, 150, 153, 193]), i32([0] * more + c.m)
    table = torch.cat([full((more, c.per), -1), i32(c.table)])
    cfg = R.page_config(1, 16, 32, c.pages, more + 3, c.per, page_bytes=c.k.stride(0), scale_bytes=c.s.stride(0))
    ws = torch.full((400 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    for size in (ws.numel(), 0):
        c.out.fill_(7)
        c.lse.fill_(7)
        R.check(R.rtcc_pages_attention(cfg, c.args[1], ptr(c.q), ptr(off), None, ptr(length), None, ptr(table), ptr(c.k), ptr(c.v),
                                       ptr(c.s), ptr(c.out), ptr(c.lse), ws.data_ptr() if size else None, size))
        c.check()


def test_write_more_sequences_than_a_grid_is_high(R):
    """70,000 sequences of one or two tokens in one call, and in two."""
    n, g = 70000, gen(11)
    new = torch.arange(n, device="cuda") % 2 + 1
    off = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), new.cumsum(0)]).int()
    tokens = int(off[-1])
    k, v = (torch.randn(tokens, 1, 16, generator=g, device="cuda").half() for _ in range(2))
    held, table = full(n, 0), torch.randperm(n, generator=g, device="cuda").int()
    pools = []
    for cuts in ((0, n), (0, n // 2, n)):
        kp, vp = (torch.zeros(n, 1, 32, 16, dtype=torch.uint8, device="cuda") for _ in range(2))
        sc = torch.zeros(n, 1, 2, 2, dtype=torch.int8, device="cuda")
        for a, b in zip(cuts, cuts[1:]):
            cfg, o = R.page_config(1, 16, 32, n, b - a, 1), off[a:b + 1].contiguous()
            t = table[a:b].contiguous()
            R.check(R.rtcc_pages_write(cfg, R.write_config(R.FP16, tokens, 2, (16, 16), (16, 16)), ptr(k), ptr(v), ptr(o), ptr(held),
                                       None, ptr(t), ptr(kp), ptr(vp), ptr(sc)))
        torch.cuda.synchronize()
        pools.append((kp, vp, sc))
    assert all(torch.equal(a, b) for a, b in zip(*pools))
    e = pools[0][2][table.long(), 0, 0, 0].double()
    first = pools[0][0][table.long(), 0, 0].view(torch.float8_e4m3fn).double() * torch.exp2(e)[:, None]
    x = k[off[:-1].long(), 0].double()
    assert bool(((first - x).abs() <= x.abs() / 16 + torch.exp2(e - 10)[:, None]).all())


@pytest.mark.parametrize("window", [0, 200])
def test_pages_workspace_of_just_the_widened_size(R, window):
    """The room that the header states, and a byte less; what lies behind it stays."""
    n, m, kv, dim = [1500, 700], [2000, 1900], 4, 64
    c = Case(n, m, 4, kv, dim, 64, window=window, sinks=10 if window else 0)
    S = max(m) if not window else 10 + window + max(n) + 192
    S = min(-(-S // 64) * 64, -(-max(m) // 64) * 64)
    room = 2 * S * kv * dim * 4 + 2 * S // 64 + 256
    ws = torch.full((room + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    c.run(R, workspace=0)
    for size in (room, room - 257 - 2 * S // 64):
        c.out.fill_(7)
        ws.fill_(0xA5)
        c.args[-2], c.args[-1] = ws.data_ptr(), size
        R.check(R.rtcc_pages_attention(*c.args, 0))
        c.check()
        assert bool((ws[size:] == 0xA5).all())
        assert size < room or bool((ws[:size // 2] != 0xA5).any())       # with less, parts of few rows may lie there


def test_pages_repeat_in_a_graph_on_a_side_stream(R):
    for n, m, window in (([1, 1], [5000, 300], 0), ([40], [900], 200), ([300], [1900], 0), ([1500], [1900], 500)):
        c = Case(n, m, 4, 2, 128, window=window)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        c.run(R, stream=s.cuda_stream)
        s.synchronize()
        c.check()
        first, lse = c.out.clone(), c.lse.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            R.check(R.rtcc_pages_attention(*c.args, torch.cuda.current_stream().cuda_stream))
        for _ in range(3):
            c.out.fill_(7)
            c.ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, first) and torch.equal(c.lse, lse)


def test_pages_without_clusters_and_given_up_waits(R):
    for workspace in (0, 32 << 20):
        try:
            assert R.rtcc_test_attention(R.TEST_NO_CLUSTERS) == R.OK
            c = Case([1], [4000], 2, 2).run(R, workspace=workspace)
        finally:
            assert R.rtcc_test_attention(0) == R.OK
        c.check()
    assert R.rtcc_memory_attention_status() == R.OK
    c = Case([1500], [1500], 4, 4)
    try:
        assert R.rtcc_test_attention(R.TEST_UNREACHABLE_WAIT) == R.OK
        c.run(R)
        assert R.rtcc_memory_attention_status() == R.E_DEVICE
    finally:
        assert R.rtcc_test_attention(0) == R.OK
    assert R.rtcc_memory_attention_status() == R.OK
    c.run(R).check()


def test_pages_untouched_tokens_and_streams(R):
    """Tokens of no sequence stay as they were; two calls on two streams do not disturb one another."""
    for n in (9, 1500):
        c = Case([5, n], [600, 1500], 4, 4, 64, 64).run(R).check()
        part = c.out[:5 + n // 2].clone()
        off, c.out[:] = i32([0, 5, 5 + n // 2]), 7.0
        c.s_d = i32(c.start)
        c.args[3], c.args[4] = ptr(off), ptr(c.s_d)
        R.check(R.rtcc_pages_attention(*c.args, 0))
        torch.cuda.synchronize()
        assert (c.out[5 + n // 2:] == 7).all() and torch.equal(c.out[:5 + n // 2], part)
        a, b = Case([n], [1500], 4, 4, 128, 32), Case([3, n], [900, 1500], 4, 2, 64, 64, "bf16", window=300, sinks=5)
        sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        for _ in range(4):
            a.run(R, stream=sa.cuda_stream)
            b.run(R, stream=sb.cuda_stream)
        a.check()
        b.check()


def test_pages_in_place_and_shared_pages(R):
    """Results over the queries; two sequences on the same pages see the same keys."""
    for n in (1, 30, 1200):
        c = Case([n, n], [1200, 1200], 4, 4, 64, 64)
        c.table[1] = list(c.table[0])
        ref = c.run(R).check().out.clone()
        q = c.q.clone(memory_format=torch.contiguous_format)
        c.q, c.out = q, q
        c.run(R)
        torch.cuda.synchronize()
        assert torch.equal(c.out, ref)


def test_pages_past_32_bits(R):
    # pages 512 MB apart: the last ones lie past 2^32 bytes
    for n in (2, 150):
        c = Case([n], [512], 1, 1, 64, 64)
        step = 1 << 29
        big = torch.empty(c.pages * step, dtype=torch.uint8, device="cuda")
        k, v = (torch.as_strided(big, (c.pages, 4096), (step, 1), at) for at in (64, 8192))
        k.copy_(c.k)
        v.copy_(c.v)
        c.k, c.v = k, v
        s = torch.empty(c.pages, step // 64, dtype=torch.int8, device="cuda")[:, :8]
        s.copy_(c.s)
        c.s = s
        c.run(R).check()
        del big


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("window", [0, 50])
def test_histories_branch_grow_and_compact(R, window):
    """Hypotheses are resampled, grow by a few tokens, attend, and are compacted now and
    then, over a dozen steps: every step's attention is that over each hypothesis's
    own tokens, followed by hand, as the pages hold them."""
    rng = random.Random(5)
    n, per, pr, pages, kv, heads, dim = 6, 8, 32, 60, 2, 4, 64
    cfg = R.page_config(kv, dim, pr, pages, n, per)
    g = gen(9)
    kp, vp = (torch.full((pages, kv, pr, dim), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
    sc = torch.full((pages, kv, pr // 16, 2), 127, dtype=torch.int8, device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    length, table = full(n, 0), full((n, per), -1)
    story = [[] for _ in range(n)]                             # per hypothesis its tokens' (k, v)
    sinks = 4
    for step in range(14):
        parent = [rng.randrange(n) for _ in range(n)] if step else list(range(n))
        keep = [len(story[p]) - rng.choice([0, 0, 0, 1, 9]) for p in parent]
        keep = [max(x, 0) for x in keep]
        new = [rng.choice([0, 1, 1, 5, 17, 33]) for _ in range(n)]
        new = [min(a, per * pr - k) for a, k in zip(new, keep)]
        held, t2, refs, out = full(n), full((n, per)), full(pages), full(n)
        src, dst, rows, short = full(n), full(n), full(n), full(1)
        pd, kd, nd = i32(parent), i32(keep), i32(new)
        R.check(R.rtcc_pages_fork(cfg, n, ptr(pd), ptr(kd), window, sinks, ptr(length), ptr(table), ptr(held), ptr(t2), ptr(refs)))
        R.check(R.rtcc_pages_extend(cfg, ptr(nd), ptr(held), ptr(t2), ptr(refs), ptr(out), ptr(src), ptr(dst), ptr(rows),
                                    ptr(short), ptr(ws), ws.numel()))
        R.check(R.rtcc_pages_copy(cfg, n, None, ptr(src), ptr(dst), ptr(rows), ptr(kp), ptr(vp), ptr(sc), pages, ptr(kp), ptr(vp),
                                  ptr(sc)))
        assert short.item() == 0 and held.tolist() == keep
        tokens = sum(new)
        k, v, q = (torch.randn(tokens, h, dim, generator=g, device="cuda").half() for h in (kv, kv, heads))
        off = i32(np.concatenate([[0], np.cumsum(new)]))
        if tokens:
            R.check(R.rtcc_pages_write(cfg, R.write_config(R.FP16, tokens, max(new), k.stride()[:2], v.stride()[:2]), ptr(k), ptr(v),
                                       ptr(off), ptr(held), ptr(out), ptr(t2), ptr(kp), ptr(vp), ptr(sc)))
        story = [story[p][:keep[i]] for i, p in enumerate(parent)]
        at = 0
        for i in range(n):
            story[i] += [(k[at + x], v[at + x]) for x in range(new[i])]
            at += new[i]
        length, table = out, t2
        assert length.tolist() == [len(x) for x in story]
        if step % 4 == 3:
            t3, r3, ms, md, mc = full((n, per)), full(pages), full(pages), full(pages), full(1)
            R.check(R.rtcc_pages_compact(cfg, ptr(table), ptr(refs), ptr(t3), ptr(r3), ptr(ms), ptr(md), ptr(mc), ptr(ws), ws.numel()))
            R.check(R.rtcc_pages_copy(cfg, pages, ptr(mc), ptr(ms), ptr(md), None, ptr(kp), ptr(vp), ptr(sc), pages, ptr(kp), ptr(vp),
                                      ptr(sc)))
            live = int((refs > 0).sum())
            assert int(t3.max()) == live - 1 and (r3[live:] == 0).all()
            table = t3
        if not tokens:
            continue
        o, lse = torch.zeros(tokens, heads, dim, device="cuda").half(), torch.zeros(tokens, heads, device="cuda")
        rc = R.page_attn_config(heads, R.FP16, tokens, q.stride()[:2], o.stride()[:2], max(new), max(length.tolist()),
                                window=window, sinks=sinks, head_dim=dim)
        R.check(R.rtcc_pages_attention(cfg, rc, ptr(q), ptr(off), ptr(held), ptr(length), None, ptr(table), ptr(kp), ptr(vp), ptr(sc),
                                       ptr(o), ptr(lse), ptr(ws), ws.numel()))
        torch.cuda.synchronize()
        rows_of, at = table.tolist(), 0
        for i in range(n):
            m = len(story[i])
            if m == 0:
                continue
            j = torch.arange(m, device="cuda")
            page = torch.tensor(rows_of[i], device="cuda")[j // pr]
            live = page >= 0
            if window == 0:
                assert bool(live.all())
            page = page.clamp(min=0)
            for h in range(kv):
                got = []
                for which, codes in ((0, kp), (1, vp)):
                    x = codes[page, h, j % pr].view(torch.float8_e4m3fn).double()
                    e = sc[page, h, j % pr // 16, which].double()
                    x = x * torch.exp2(e)[:, None]
                    # what the pages hold is the tokens: e4m3 numbers are good to 2^-4 of themselves or half a step of 2^(e - 9),
                    # and may have been rounded again once for every rise of their block's exponent, which halves nothing
                    true = torch.stack([t[which][h] for t in story[i]]).double()
                    err = (x - true).abs()
                    lim = true.abs() * 2.0 ** -3 + torch.exp2(e - 9)[:, None]
                    assert bool((err <= lim)[live].all())
                    got.append(torch.where(live[:, None], x, 0.0))
                for r in range(new[i]):
                    p = m - new[i] + r
                    see = (j <= p) & live
                    if window:
                        see = see & ((j > p - window) | (j < sinks))
                    for hq in range(h * 2, h * 2 + 2):
                        x = torch.where(see, got[0] @ q[at + r, hq].double() / 8, -math.inf)
                        w = torch.softmax(x, 0)
                        want, A = w @ got[1], w @ got[1].abs()
                        assert bool(((o[at + r, hq].double() - want).abs() <= (2.0 ** -10 + 2.0 ** -15) * A + 2.0 ** -25).all())
            at += new[i]
