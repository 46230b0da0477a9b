"""Token memory on the GPU against plain float64 forms.

Tolerances.  u is the storage type's unit roundoff (2^-11 fp16, 2^-8 bf16).
prepare: one rounding of the result, and float32 arithmetic on the way: a few
roundings of 2^-24 of the pair's length, and an angle good to 2^-24 turns
(4e-7): |err| <= u |y| + 2^-19 |pair| (+ the type's smallest subnormal).
attention: with A = sum_j p_j |v_j|, rounding the probabilities costs u A, the
result's rounding u |out| <= u A, a score error d costs 2 d A, and the float32
sums 2^-20 A.  d: float32 sums of head_dim products (2^-23 of the largest sum of
their magnitudes times sqrt(head_dim)), tanh to 4e-7 of the cap, the bias to
2^-22 of its size, the exponential to 2^-21.
"""
import math

import numpy as np
import pytest

from tests import gpu_util as U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -133}


@pytest.fixture(scope="module")
def R():
    return U.load()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def f64(t):
    return t.double().cpu().numpy()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

def append_reference(new, held, slot, capacity, n_tokens):
    n = len(new)
    off, rows, seq, pos, begin, end, length = [0], [], [], [], [], [], []
    for s in range(n):
        take = min(max(new[s], 0), n_tokens - off[-1])
        h = min(max(held[s], 0), capacity)
        ok = slot[s] >= 0 and (slot[s] + 1) * capacity < 2 ** 31
        for i in range(take):
            rows.append(slot[s] * capacity + h + i if ok and h + i < capacity else -1)
            seq.append(s)
            pos.append(h + i)
        off.append(off[-1] + take)
        length.append(min(capacity, h + take))
        begin.append(slot[s] * capacity if ok else 0)
        end.append(begin[-1] + (length[-1] if ok else 0))
    pad = [-1] * (n_tokens - len(rows))
    return off, rows + pad, seq + pad, pos + pad, begin, end, length


def run_append(R, new, held, slot, capacity, n_tokens, optional=True):
    n = len(new)
    e = lambda k: torch.full((k,), -77, dtype=torch.int32, device="cuda")  # noqa: E731
    off, rows, seq, pos, begin, end, length = e(n + 1), e(n_tokens), e(n_tokens), e(n_tokens), e(n), e(n), e(n)
    a, b, c = i32(new), i32(held), None if slot is None else i32(slot)
    p = lambda t: t.data_ptr() if t is not None and t.numel() else None  # noqa: E731
    s = R.rtcc_memory_append(n, capacity, n_tokens, p(a), p(b), p(c), p(off), p(rows), p(seq) if optional else None,
                             p(pos) if optional else None, p(begin), p(end), p(length), 0)
    assert s == R.OK
    torch.cuda.synchronize()
    return [t.cpu().tolist() for t in (off, rows, seq, pos, begin, end, length)]


@pytest.mark.parametrize("n_seqs,most,capacity,spare", [
    (1, 1, 1, 0), (1, 5000, 4096, 7), (2, 0, 10, 3), (3, 1, 5, -1), (61, 1, 100, 0), (513, 7, 9, -20), (2048, 40, 33, 11),
    (16384, 3, 20, 0)])
def test_append_matches_the_loop(R, n_seqs, most, capacity, spare):
    rng = np.random.default_rng(n_seqs + most)
    new = rng.integers(0, most + 1, n_seqs)
    held = rng.integers(0, capacity + 1, n_seqs)
    slot = rng.permutation(n_seqs)
    n_tokens = max(0, int(new.sum()) + spare)            # a negative spare: some tokens have no place
    want = append_reference(new.tolist(), held.tolist(), slot.tolist(), capacity, n_tokens)
    assert run_append(R, new, held, slot, capacity, n_tokens) == [list(x) for x in want]


def test_append_odd_inputs(R):
    # negative counts, held past the capacity, a negative slot, a slot past 2^31 rows, no slot map
    new, held, slot = [3, -4, 2, 2, 1], [-5, 9, 99, 1, 0], [0, 1, 2, -1, 400000000]
    want = append_reference(new, held, slot, 8, 10)
    assert run_append(R, new, held, slot, 8, 10) == [list(x) for x in want]
    want = append_reference(new, held, list(range(5)), 8, 10)
    got = run_append(R, new, held, None, 8, 10, optional=False)
    assert got[0] == want[0] and got[1] == want[1] and got[4:] == [list(x) for x in want[4:]]
    assert got[2] == [-77] * 10 and got[3] == [-77] * 10
    assert run_append(R, [2 ** 31 - 1, 2 ** 31 - 1, 5], [0, 0, 0], None, 4, 6)[0] == [0, 6, 6, 6]
    assert run_append(R, [], [], None, 4, 3)[:4] == [[0], [-1] * 3, [-1] * 3, [-1] * 3]


# ---------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------

def turn_reference(x, gain, pos, axis_pairs, interleaved, norm, theta, eps):
    """(result, length of each channel's pair) in float64."""
    x = np.array(x, dtype=np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        x = x * gain
    rot = sum(axis_pairs)
    size = np.abs(x)
    m = 0
    y = x.copy()
    for a, n in enumerate(axis_pairs):
        for i in range(n):
            ang = pos[:, a].astype(np.float64) * theta ** (-i / n)
            c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
            u, v = (2 * m, 2 * m + 1) if interleaved else (m, m + rot)
            y[..., u] = x[..., u] * c - x[..., v] * s
            y[..., v] = x[..., u] * s + x[..., v] * c
            size[..., u] = size[..., v] = np.hypot(x[..., u], x[..., v])
            m += 1
    return y, size


def check_turned(got, x, gain, pos, dtype, what, **kw):
    want, size = turn_reference(x, gain, pos, **kw)
    lim = ROUND[dtype] * np.abs(want) + 2.0 ** -19 * size + TINY[dtype]
    err = np.abs(f64(got) - want)
    assert (err <= lim).all(), (what, float((err / lim).max()))


@pytest.mark.parametrize("dim,heads,kv,pairs", [
    (8, 1, 1, (4, 0, 0)), (8, 3, 1, (1, 1, 1)), (16, 5, 5, (0, 3, 4)), (24, 2, 1, (5, 0, 7)), (32, 12, 3, (4, 6, 6)),
    (40, 7, 7, (3, 7, 2)), (64, 6, 6, (8, 12, 12)), (64, 1, 1, (0, 0, 0)), (72, 4, 2, (36, 0, 0)), (80, 10, 5, (4, 9, 11)),
    (96, 8, 1, (16, 16, 16)), (128, 32, 8, (64, 0, 0)), (128, 3, 3, (0, 21, 22))])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_prepare_matches_float64(R, dim, heads, kv, pairs, interleaved, dtype):
    g = gen(dim * 7 + heads)
    n, n_rows = 37, 50
    dt = DT[dtype]
    packed = dim % 16 == 0
    x = (torch.randn(n, heads + 2 * kv, dim, generator=g, device="cuda")
         * torch.logspace(-2, 2, heads + 2 * kv, device="cuda")[:, None]).to(dt)
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    gains = [1 + 0.3 * torch.randn(dim, generator=g, device="cuda") for _ in range(2)] if heads != 6 else [None, None]
    pos = torch.randint(-300, 100000, (n, 3), generator=g, device="cuda").float()
    pos[:, 1:] *= 0.013
    rows = torch.randperm(n_rows, generator=g, device="cuda")[:n].int()
    rows[3], rows[11], rows[20] = -1, n_rows, 2 ** 31 - 1
    # memories wider than they need be: a stride of their own, guarded
    km = torch.full((n_rows, kv, dim + 8), 9.0, device="cuda", dtype=dt)
    vm = torch.full((n_rows, 2 * kv, dim), 9.0, device="cuda", dtype=dt)
    qo = torch.full((n, heads, dim), 9.0, device="cuda", dtype=dt)
    coord = torch.full((n_rows, 2), 9.0, device="cuda")
    kw = dict(axis_pairs=pairs, interleaved=interleaved, norm=True, theta=10000.0, eps=1e-6)
    cfg = R.prepare_config(heads, kv, dim, R.BF16 if dtype == "bf16" else R.FP16, n, n_rows, q.stride()[:2],
                           k.stride()[:2], v.stride()[:2], qo.stride()[:2], km.stride()[:2], vm.stride()[:2], **kw)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    R.check(R.rtcc_qkv_prepare(cfg, ptr(q), ptr(k), ptr(v), ptr(gains[0]), ptr(gains[1]), ptr(pos), ptr(rows), ptr(qo),
                               ptr(km), ptr(vm), ptr(coord), 0))
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    gn = [None if t is None else f64(t) for t in gains]
    check_turned(qo, f64(q), gn[0], p, dtype, "q", **kw)
    r = rows.cpu().numpy()
    live = np.flatnonzero((r >= 0) & (r < n_rows))
    at = torch.tensor(r[live], dtype=torch.long, device="cuda")
    check_turned(km[at][..., :dim], f64(k)[live], gn[1], p[live], dtype, "k", **kw)
    assert torch.equal(vm[at][:, :kv], v[torch.tensor(live, device="cuda")])
    np.testing.assert_array_equal(coord[at].cpu().numpy(), p[live][:, 1:])
    rest = torch.ones(n_rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (km[rest] == 9).all() and (vm[rest] == 9).all() and (coord[rest] == 9).all()
    assert (km[..., dim:] == 9).all() and (vm[:, kv:] == 9).all()


@pytest.mark.parametrize("n", [0, 1, 2, 5000])
@pytest.mark.parametrize("interleaved", [False, True])
def test_prepare_in_place_without_norm_queries_only(R, n, interleaved):
    g = gen(n + 5)
    q = torch.randn(n, 3, 48, generator=g, device="cuda").half()
    keep, pos = q.clone(), torch.rand(n, 3, generator=g, device="cuda") * 50
    kw = dict(axis_pairs=(7, 5, 9), interleaved=interleaved, norm=False, theta=500.0, eps=0.0)
    st = (144, 48)
    cfg = R.prepare_config(3, 1, 48, R.FP16, n, 0, st, st, st, st, st, st, **kw)
    R.check(R.rtcc_qkv_prepare(cfg, q.data_ptr(), None, None, None, None, pos.data_ptr(), None, q.data_ptr(), None, None,
                               None, 0))
    torch.cuda.synchronize()
    if n:
        check_turned(q, f64(keep), None, pos.cpu().numpy(), "fp16", "q", **kw)


def test_prepare_extremes(R):
    # an all-zero head, the type's largest values, non-finite channels in one head only, far positions
    n, heads, dim = 6, 4, 64
    q = torch.randn(n, heads, dim, generator=gen(9), device="cuda").half()
    q[0, 0] = 0
    q[1, 1] = 65504
    q[2, 2, 5] = float("inf")
    q[3, 3, 7] = float("nan")
    pos = torch.tensor([[2.0 ** 24 - 1, -123456.75, 0.001]] * n, device="cuda")
    out = torch.empty_like(q)
    kw = dict(axis_pairs=(10, 11, 11), interleaved=False, norm=True, theta=10000.0, eps=1e-6)
    st = (heads * dim, dim)
    cfg = R.prepare_config(heads, 1, dim, R.FP16, n, 0, st, st, st, st, st, st, **kw)
    R.check(R.rtcc_qkv_prepare(cfg, q.data_ptr(), None, None, None, None, pos.data_ptr(), None, out.data_ptr(), None,
                               None, None, 0))
    torch.cuda.synchronize()
    fine = torch.isfinite(q).all(-1).cpu().numpy()
    want, size = turn_reference(np.where(fine[..., None], f64(q), 0.0), None, pos.cpu().numpy(), **kw)
    err = np.abs(f64(out) - want)
    assert (err <= 2.0 ** -11 * np.abs(want) + 2.0 ** -19 * size + TINY["fp16"])[fine].all()
    assert not torch.isfinite(out[3, 3]).any() and (out[0, 0] == 0).all()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

class Case:
    """Random sequences over a memory; rows that nobody sees hold NaN."""

    def __init__(self, n, m, heads=2, kv=1, dim=64, dtype="fp16", causal=False, prefix=None, cap=0.0, dist=False,
                 slot_rows=0, absent=(), gap=0, shared=False, seed=0, spread=1.0, lse=True, q_wide=0, k_wide=0):
        g = gen(seed + 1000)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.n, self.m, self.heads, self.kv, self.dim, self.dtype = list(n), list(m), heads, kv, dim, dtype
        self.causal, self.prefix, self.cap, self.dist, self.slot_rows, self.absent = causal, prefix, cap, dist, slot_rows, absent
        dt = DT[dtype]
        self.begin, at = [], gap
        for x in m:
            self.begin.append(gap if shared else at)
            at += x + gap
        self.rows = max([b + x for b, x in zip(self.begin, m)] + [0]) + gap
        self.tokens = sum(n)
        q = (spread * rand(self.tokens, heads, dim + q_wide)).to(dt)
        k, v = rand(self.rows, kv, dim + k_wide).to(dt), rand(self.rows, kv, dim + k_wide).to(dt)
        self.q, self.k, self.v = q[..., :dim], k[..., :dim], v[..., :dim]
        seen = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        for b, x in zip(self.begin, m):
            seen[b:b + x] = True
        self.present = None
        if slot_rows:
            n_slots = max(1, -(-self.rows // slot_rows))
            self.present = torch.ones(n_slots, dtype=torch.int32, device="cuda")
            for s in absent:
                self.present[s] = 0
                seen[s * slot_rows:(s + 1) * slot_rows] = False
        k[~seen] = float("nan")
        v[~seen] = float("inf")
        self.slopes = self.q_pos = self.k_pos = None
        if dist:
            self.slopes = 0.3 * 2.0 ** -torch.arange(heads, device="cuda").float()
            self.q_pos = 20 * torch.rand(self.tokens, 3, generator=g, device="cuda")
            self.k_pos = 20 * torch.rand(self.rows, 2, generator=g, device="cuda")
            self.k_pos[~seen] = float("nan")
        self.out = torch.full((self.tokens, heads, dim), 7.0, device="cuda", dtype=dt)
        self.lse = torch.full((self.tokens, heads), 7.0, device="cuda") if lse else None
        self.scale = 1 / math.sqrt(dim)

    def run(self, R, workspace=32 << 20, max_q=None, max_k=None, stream=0, off=None, span=None):
        p = lambda t: None if t is None or not t.numel() else t.data_ptr()  # noqa: E731
        self.off_d = off if off is not None else i32(np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32))
        self.b_d = i32(self.begin)
        self.e_d = i32([b + x for b, x in zip(self.begin, self.m)])
        self.p_d = None if self.prefix is None else i32(self.prefix)
        self.ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        cfg = R.attn_config(self.heads, self.kv, self.dim, R.BF16 if self.dtype == "bf16" else R.FP16, self.tokens,
                            self.rows, self.q.stride()[:2], self.k.stride()[:2], self.v.stride()[:2], self.out.stride()[:2],
                            len(self.n), max(self.n + [0]) if max_q is None else max_q,
                            max(self.m + [0]) if max_k is None else max_k, causal=self.causal,
                            n_slots=0 if self.present is None else self.present.numel(), slot_rows=self.slot_rows,
                            q_pos_row=3, scale=self.scale, cap=self.cap)
        R.check(R.rtcc_memory_attention(cfg, p(self.q), p(self.k), p(self.v), p(self.off_d), p(self.b_d), p(self.e_d),
                                        p(self.p_d), p(self.present), p(self.slopes), p(self.q_pos), p(self.k_pos),
                                        p(self.out), p(self.lse), self.ws.data_ptr() if workspace else None, workspace,
                                        stream))
        return self

    def visible(self, s):
        n, m, b = self.n[s], self.m[s], self.begin[s]
        see = np.ones((n, m), dtype=bool)
        if self.causal:
            i, j = np.arange(n)[:, None], np.arange(m)[None]
            see = (j <= i + m - n) | (j < (self.prefix[s] if self.prefix is not None else 0))
        if self.slot_rows:
            see = see & (self.present.cpu().numpy()[(b + np.arange(m)) // self.slot_rows] != 0)[None]
        return see

    def check(self):
        torch.cuda.synchronize()
        u, at = ROUND[self.dtype], 0
        q, k, v = self.q.double(), self.k.double(), self.v.double()
        for s, (n, m, b) in enumerate(zip(self.n, self.m, self.begin)):
            see = torch.tensor(self.visible(s), device="cuda").reshape(n, m)
            for h in range(self.heads):
                kh = h // (self.heads // self.kv)
                # rows nobody sees hold NaN: the reference leaves them out
                kk = torch.where(see.any(0)[:, None], k[b:b + m, kh], 0.0)
                vv = torch.where(see.any(0)[:, None], v[b:b + m, kh], 0.0)
                qq = q[at:at + n, h]
                x = self.scale * (qq @ kk.T)
                size = self.scale * float((qq.abs() @ kk.abs().T).max()) if n and m else 0.0
                if self.cap:
                    x = self.cap * torch.tanh(x / self.cap)
                bias = 0.0
                if self.dist:
                    kp = torch.nan_to_num(self.k_pos[b:b + m].double())
                    d = (self.q_pos[at:at + n, None, :2].double() - kp[None]).abs().sum(-1)
                    x = x - float(self.slopes[h]) * d
                    bias = float(self.slopes[h]) * float(d.max()) if d.numel() else 0.0
                x = torch.where(see, x, -math.inf)
                lse = torch.logsumexp(x, 1) if m else torch.full((n,), -math.inf, device="cuda", dtype=torch.float64)
                p = torch.where(see, torch.exp(x - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
                want, A = p @ vv, p @ vv.abs()
                d = 2.0 ** -23 * math.sqrt(self.dim) * size + 4e-7 * self.cap + 2.0 ** -22 * bias + 2.0 ** -21
                got = self.out[at:at + n, h].double()
                err = (got - want).abs()
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


LENGTHS = [
    # (tokens, keys) of the sequences
    ([1], [1]), ([1], [0]), ([1], [63]), ([1], [129]), ([2], [5000]), ([16], [257]), ([17], [1000]), ([127], [127]),
    ([128], [128]), ([129], [385]), ([257], [1023]), ([300], [20000]), ([1, 1, 1, 1], [1, 0, 777, 4096]),
    ([0, 3, 0, 40], [10, 3, 0, 200]), ([5, 64, 200, 1], [0, 64, 333, 1]),
]


@pytest.mark.parametrize("n,m", LENGTHS)
@pytest.mark.parametrize("dim,heads,kv", [(64, 2, 2), (128, 4, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_lengths(R, n, m, dim, heads, kv, causal):
    Case(n, m, heads=heads, kv=kv, dim=dim, dtype="bf16" if causal else "fp16", causal=causal, gap=3).run(R).check()


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 56, 64, 72, 96, 104, 120, 128])
@pytest.mark.parametrize("n,m", [([1, 1], [300, 70]), ([150, 3], [333, 90])])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_head_sizes(R, dim, n, m, dtype):
    Case(n, m, heads=3, kv=3, dim=dim, dtype=dtype, dist=dim % 16 == 0, cap=20.0 if dim % 24 == 0 else 0.0, gap=5).run(R).check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (5, 5), (6, 2), (8, 1), (20, 1), (40, 2)])
@pytest.mark.parametrize("n,m", [([1, 1, 1], [700, 1, 33]), ([4, 9], [200, 100]), ([200], [260])])
def test_attention_head_groups(R, heads, kv, n, m):
    Case(n, m, heads=heads, kv=kv, dim=64, causal=True, prefix=[7] * len(n), seed=heads).run(R).check()


@pytest.mark.parametrize("cap,dist", [(0.0, False), (30.0, False), (2.0, False), (0.0, True), (50.0, True)])
@pytest.mark.parametrize("n,m", [([1], [3000]), ([33], [500]), ([300], [600])])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_scores(R, cap, dist, n, m, dim):
    # widely spread scores: the maximum moves often, and the cap works
    Case(n, m, heads=2, kv=1, dim=dim, cap=cap, dist=dist, spread=6.0, dtype="bf16").run(R).check()


@pytest.mark.parametrize("n,m", [([1, 1], [500, 40]), ([30, 200], [64, 130]), ([256], [100]), ([400], [700])])
def test_attention_causal_prefix_and_empty_rows(R, n, m):
    # sequences with more tokens than keys: their first tokens see nothing but the prefix
    for prefix in (None, [0] * len(n), [5] * len(n), [10 ** 6] * len(n)):
        c = Case(n, m, heads=2, kv=2, causal=True, prefix=prefix, gap=9, seed=len(n)).run(R)
        if prefix == [10 ** 6] * len(n):
            c.prefix = list(m)                       # cut to the span
        c.check()


@pytest.mark.parametrize("slot_rows,absent", [(100, (1,)), (100, (0, 2, 3)), (37, (0, 5, 9)), (1, tuple(range(0, 60, 3))),
                                              (130, (0, 1, 2, 3)), (128, (1, 2))])
@pytest.mark.parametrize("n", [1, 20, 300])
def test_attention_absent_slots(R, slot_rows, absent, n):
    m = min(slot_rows * 64, 400) if slot_rows > 1 else 60
    absent = [s for s in absent if s * slot_rows < m]
    for dim in (64, 128):
        Case([n], [m], heads=2, kv=1, dim=dim, slot_rows=slot_rows, absent=absent, dist=dim == 64, cap=10.0).run(R).check()


@pytest.mark.parametrize("n", [1, 40, 260])
def test_attention_shared_rows_and_strides(R, n):
    # several sequences over the same rows; heads and rows with strides of their own
    c = Case([n, n, 2], [900, 500, 900], heads=4, kv=2, dim=64, shared=True, q_wide=16, k_wide=64, causal=True)
    wide = torch.full((c.tokens, 4, 80), 7.0, device="cuda", dtype=torch.float16)
    c.out = wide[..., :64]
    c.run(R).check()
    assert (wide[..., 64:] == 7).all()


@pytest.mark.parametrize("n,m", [([1], [9000]), ([3, 1], [7000, 20]), ([100], [6000])])
def test_attention_split_and_hints(R, n, m):
    """Results hold with and without a workspace, with one too small, and with
    hints that are too small or too large."""
    for kw in (dict(workspace=0), dict(workspace=20000), dict(), dict(max_q=1, max_k=1), dict(max_q=1, max_k=100),
               dict(max_q=10 ** 6, max_k=10 ** 9)):
        Case(n, m, heads=4, kv=2, dim=128, causal=True, dtype="bf16").run(R, **kw).check()


@pytest.mark.parametrize("dim", [64, 80])
@pytest.mark.parametrize("n,m", [([1], [130]), ([1], [1025]), ([3], [2049]), ([5], [4097]), ([1, 1, 1], [900, 0, 31]),
                                 ([2, 0, 4, 1], [1, 700, 2000, 650])])
def test_attention_joined_inside_clusters(R, n, m, dim):
    """Few chunks: the blocks of a cluster join them, with and without a
    workspace, over chunks that are empty, rows past the last and absent slots."""
    for kw in (dict(heads=8, kv=2), dict(heads=6, kv=6, slot_rows=150, absent=(0, 2), cap=30.0, dist=True)):
        if kw.get("absent"):                     # slots that the memory has
            kw["absent"] = [a for a in kw["absent"] if a * 150 < sum(m)]
        c = Case(n, m, dim=dim, causal=True, gap=3, **kw)
        for run in (dict(), dict(workspace=0), dict(max_k=60 * 64)):
            c.out.fill_(7.0)
            c.run(R, **run).check()


def test_attention_repeats_bit_for_bit(R):
    a = Case([1, 30], [9000, 4000], heads=4, kv=2, dim=64, causal=True).run(R).check()
    b = Case([1, 30], [9000, 4000], heads=4, kv=2, dim=64, causal=True).run(R)
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


def test_attention_without_lse_and_untouched_tokens(R):
    c = Case([3, 50], [40, 700], lse=False)
    c.run(R).check()
    # offsets that leave the last tokens to no sequence, and offsets past the arrays
    c = Case([3, 50], [40, 700])
    c.run(R, off=i32([0, 3, 43]))
    torch.cuda.synchronize()
    assert (c.out[43:] == 7).all() and not (c.out[:43] == 7).all()
    c = Case([3, 50], [40, 700])
    c.run(R, off=i32([-5, 3, 10 ** 9])).check()


def test_attention_in_place(R):
    for n, m in (([1, 4], [3000, 100]), ([300], [400])):
        c = Case(n, m, heads=4, kv=2, dim=64)
        ref = Case(n, m, heads=4, kv=2, dim=64).run(R).check()
        c.out = c.q
        c.run(R)
        torch.cuda.synchronize()
        assert torch.equal(c.out, ref.out)


def test_attention_visible_non_finite_stays_in_its_rows(R):
    for n in (1, 200):
        c = Case([n, 5], [300, 300], heads=2, kv=2)
        c.q[0, 0, 3] = float("nan")
        ref = Case([n, 5], [300, 300], heads=2, kv=2).run(R).check()
        c.run(R)
        torch.cuda.synchronize()
        assert torch.isnan(c.out[0, 0]).all() and torch.isnan(c.lse[0, 0])
        same = torch.ones(n + 5, 2, dtype=torch.bool, device="cuda")
        same[0, 0] = False
        assert torch.equal(c.out[same], ref.out[same]) and torch.equal(c.lse[same], ref.lse[same])


def test_attention_offsets_past_32_bits(R):
    # rows a megabyte apart: the last row lies past 2^31 elements
    for n in (2, 150):
        c = Case([n], [2304], heads=1, kv=1, dim=64)
        big = torch.empty((2304, 1 << 20), dtype=torch.float16, device="cuda")
        k, v = big[:, 64:128], big[:, 4096:4160]
        k.copy_(c.k[:, 0])
        v.copy_(c.v[:, 0])
        c.k, c.v = k.unsqueeze(1), v.unsqueeze(1)
        c.run(R).check()


def test_attention_on_a_side_stream_and_in_a_graph(R):
    for n, m in (([1, 1], [5000, 300]), ([200], [900])):
        s = torch.cuda.Stream()
        c = Case(n, m, heads=2, kv=1, dim=128)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            c.run(R, stream=s.cuda_stream)
        s.synchronize()
        c.check()
        first = c.out.clone()
        graph = torch.cuda.CUDAGraph()
        keep = (c.off_d, c.b_d, c.e_d, c.ws)             # the capture's inputs
        cfg = R.attn_config(2, 1, 128, R.FP16, c.tokens, c.rows, c.q.stride()[:2], c.k.stride()[:2], c.v.stride()[:2],
                            c.out.stride()[:2], len(n), max(n), max(m))
        with torch.cuda.graph(graph):
            R.check(R.rtcc_memory_attention(cfg, c.q.data_ptr(), c.k.data_ptr(), c.v.data_ptr(), keep[0].data_ptr(),
                                            keep[1].data_ptr(), keep[2].data_ptr(), None, None, None, None, None,
                                            c.out.data_ptr(), c.lse.data_ptr(), keep[3].data_ptr(), keep[3].numel(),
                                            torch.cuda.current_stream().cuda_stream))
        for _ in range(3):
            c.out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, first)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def test_append_prepare_attend_step_by_step(R):
    """Sequences fed in bursts give, token for token, what one pass over the
    whole sequences gives."""
    g = gen(3)
    seqs, heads, kv, dim, capacity, total = 3, 4, 2, 64, 64, [50, 17, 64]
    pairs = (32, 0, 0)
    x = [torch.randn(t, heads + 2 * kv, dim, generator=g, device="cuda").half() for t in total]
    rows = seqs * capacity
    km = torch.full((rows, kv, dim), float("nan"), device="cuda", dtype=torch.float16)
    vm = torch.full_like(km, float("nan"))
    held = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    slot = i32([2, 0, 1])
    outs = [[] for _ in range(seqs)]
    done = [0] * seqs
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(0)
    while done != total:
        new = [min(int(rng.integers(0, 30)), t - d) for t, d in zip(total, done)]
        n = sum(new)
        e = lambda k: torch.empty(max(k, 1), dtype=torch.int32, device="cuda")  # noqa: E731
        off, row, pos, begin, end, length = e(seqs + 1), e(n), e(n), e(seqs), e(seqs), e(seqs)
        fresh = i32(new)
        R.check(R.rtcc_memory_append(seqs, capacity, n, fresh.data_ptr(), held.data_ptr(), slot.data_ptr(),
                                     off.data_ptr(), row.data_ptr(), None, pos.data_ptr(), begin.data_ptr(),
                                     end.data_ptr(), length.data_ptr()))
        if n:
            tok = torch.cat([x[s][done[s]:done[s] + new[s]] for s in range(seqs)])
            p3 = torch.zeros(n, 3, device="cuda")
            p3[:, 0] = pos[:n].float()
            q = torch.empty(n, heads, dim, device="cuda", dtype=torch.float16)
            st = tok.stride()[:2]
            cfg = R.prepare_config(heads, kv, dim, R.FP16, n, rows, st, st, st, q.stride()[:2], km.stride()[:2],
                                   vm.stride()[:2], pairs)
            R.check(R.rtcc_qkv_prepare(cfg, tok.data_ptr(), tok[:, heads:].data_ptr(), tok[:, heads + kv:].data_ptr(),
                                       None, None, p3.data_ptr(), row.data_ptr(), q.data_ptr(), km.data_ptr(),
                                       vm.data_ptr(), None))
            out = torch.empty_like(q)
            a = R.attn_config(heads, kv, dim, R.FP16, n, rows, q.stride()[:2], km.stride()[:2], vm.stride()[:2],
                              out.stride()[:2], seqs, max(new), capacity, causal=True)
            R.check(R.rtcc_memory_attention(a, q.data_ptr(), km.data_ptr(), vm.data_ptr(), off.data_ptr(),
                                            begin.data_ptr(), end.data_ptr(), None, None, None, None, None,
                                            out.data_ptr(), None, ws.data_ptr(), ws.numel()))
            torch.cuda.synchronize()
            at = 0
            for s in range(seqs):
                outs[s].append(out[at:at + new[s]])
                at += new[s]
        held = length.clone()
        done = [d + k for d, k in zip(done, new)]
    for s in range(seqs):
        got = f64(torch.cat(outs[s]))
        pos = np.zeros((total[s], 3))
        pos[:, 0] = np.arange(total[s])
        kw = dict(axis_pairs=pairs, interleaved=False, norm=True, theta=10000.0, eps=1e-6)
        xs = f64(x[s])
        q = turn_reference(xs[:, :heads], None, pos, **kw)[0]
        k = turn_reference(xs[:, heads:heads + kv], None, pos, **kw)[0]
        # q and k are rounded to fp16: a relative 2^-11 each of every product, on scores of at most
        # sqrt(dim) = 8 after the norm: 2 * 2^-11 * 8 on a score, besides the attention's own errors
        for h in range(heads):
            sc = q[:, h] @ k[:, h // 2].T / 8.0
            sc[np.triu_indices(total[s], 1)] = -np.inf
            p = np.exp(sc - sc.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            v = xs[:, heads + kv + h // 2]
            lim = (2 * 2.0 ** -11 + 2 * (2 * 2.0 ** -11 * 8)) * (p @ np.abs(v)) + 1e-6
            assert (np.abs(got[:, h] - p @ v) <= lim).all()


def test_token_fusion_of_a_frame(R):
    """The example's whole path on a small frame, against the formula in float64
    on the frame's own feature maps.  q and k carry one rounding each (u relative
    of every product: 2 u of a score's largest magnitude, sqrt(dim) after the
    norm), besides the attention's own errors."""
    from paper_2608_08330_gb300 import token_fusion as F
    for absent in ((), (1,)):
        cfg, maps = F.frame_maps("tiny", 3, absent)
        cell = cfg.pillar * cfg.feat_stride
        out, lse = F.fuse(maps, cfg.dtype, cfg.feat_h, cfg.feat_w, cell)
        cells, (heads, dim) = cfg.feat_h * cfg.feat_w, F.head_layout(cfg.feat_ch)
        kw = dict(axis_pairs=F.axis_pairs(dim), interleaved=False, norm=True, theta=F.THETA, eps=F.EPS)
        x = [U.u16_to_f64(m, cfg.dtype).reshape(cells, heads, dim) for m in maps if m is not None]
        pos = [F.positions(k, cfg.feat_h, cfg.feat_w, cell) for k, m in enumerate(maps) if m is not None]
        q = turn_reference(x[0], None, pos[0], **kw)[0]
        k = np.concatenate([turn_reference(a, None, p, **kw)[0] for a, p in zip(x, pos)])
        v, yx = np.concatenate(x), np.concatenate(pos)[:, 1:].astype(np.float64)
        u = ROUND[cfg.dtype]
        for i in np.linspace(0, cells - 1, 40).astype(int):
            for h in range(heads):
                s = k[:, h] @ q[i, h] / math.sqrt(dim)
                s = F.CAP * np.tanh(s / F.CAP) - float(F.slopes(heads)[h]) * np.abs(yx - yx[i]).sum(1)
                p = np.exp(s - s.max())
                want, A = p @ v[:, h] / p.sum(), p @ np.abs(v[:, h]) / p.sum()
                d = 2 * u * math.sqrt(dim)
                assert (np.abs(f64(out[i, h]) - want) <= (2 * u + 2 * d) * A + 1e-6).all()
                assert abs(float(lse[i, h]) - (np.log(p.sum()) + s.max())) <= d + 1e-5


def test_attention_status_is_clean(R):
    Case([300], [500], heads=2, kv=2).run(R).check()
    assert R.rtcc_memory_attention_status() == R.OK
