"""Token memory at its edges: sizes near 2^31, scores and caps far from the usual
ones, non-finite values, slots that fill up, hints that are too small, and what
happens when a launch or a wait fails.

Tolerances are those of test_gpu_tokens.py (u: the storage type's unit roundoff,
d: a score's error, A = sum_j p_j |v_j|), unless a test derives its own.
"""
import math

import numpy as np
import pytest

from tests import gpu_util as U
from tests.test_gpu_tokens import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def R():
    return U.load()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

def test_append_token_places_up_to_2_to_the_31(R):
    """The last token places lie within one grid's stride of 2^31: the walk over
    them must end there."""
    n, guard = 2 ** 31 - 1, 64
    buf = torch.full((n + 2 * guard + 1,), -77, dtype=torch.int32, device="cuda")
    rows = buf[guard:guard + n]
    e = lambda k: torch.full((k,), -77, dtype=torch.int32, device="cuda")  # noqa: E731
    off, begin, end, length = e(3), e(2), e(2), e(2)
    new, held = i32([3, 2]), i32([1, 0])
    assert R.rtcc_memory_append(2, 10, n, new.data_ptr(), held.data_ptr(), None, off.data_ptr(), rows.data_ptr(), None,
                                None, begin.data_ptr(), end.data_ptr(), length.data_ptr()) == R.OK
    torch.cuda.synchronize()
    assert off.tolist() == [0, 3, 5] and rows[:5].tolist() == [1, 2, 3, 10, 11]
    for lo in range(5, n, 1 << 28):
        assert bool((rows[lo:lo + (1 << 28)] == -1).all()), lo
    assert bool((buf[:guard] == -77).all()) and bool((buf[guard + n:] == -77).all())


# ---------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 700])
@pytest.mark.parametrize("dim,pairs", [(64, (8, 12, 12)), (8, (0, 0, 0)), (80, (3, 4, 4))])
def test_prepare_writes_coordinates_alone(R, n, dim, pairs):
    pos = torch.rand(n, 3, device="cuda")
    rows = torch.randperm(n + 5, device="cuda")[:n].int()
    rows[0] = -1
    coord = torch.full((n + 5, 2), 9.0, device="cuda")
    cfg = R.prepare_config(4, 2, dim, R.FP16, n, n + 5, *[(4 * dim, dim)] * 6, pairs)
    R.check(R.rtcc_qkv_prepare(cfg, None, None, None, None, None, pos.data_ptr(), rows.data_ptr(), None, None, None,
                               coord.data_ptr()))
    torch.cuda.synchronize()
    want = torch.full_like(coord, 9.0)
    want[rows[1:].long()] = pos[1:, 1:]
    assert torch.equal(coord, want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(64, (8, 4, 4)), (64, (5, 3, 3)), (64, (0, 0, 0)), (40, (1, 0, 6)), (128, (0, 3, 0))])
def test_prepare_leaves_unturned_channels_alone(R, interleaved, dim, pairs):
    """Channels past the turned pairs keep their bits without a norm, beside infinities and NaN too."""
    n, rot = 9, 2 * sum(pairs)
    g = torch.Generator(device="cuda")
    g.manual_seed(dim + rot)
    q = torch.randn(n, 2, dim, generator=g, device="cuda").half()
    for e in range(rot, dim, 3):
        q[e % n, e % 2, e] = float("inf") if e % 4 else float("nan")
    pos, out = 9 * torch.rand(n, 3, generator=g, device="cuda"), torch.empty_like(q)
    cfg = R.prepare_config(2, 1, dim, R.FP16, n, 0, *[(2 * dim, dim)] * 6, pairs, interleaved=interleaved, norm=False)
    R.check(R.rtcc_qkv_prepare(cfg, q.data_ptr(), None, None, None, None, pos.data_ptr(), None, out.data_ptr(), None, None,
                               None))
    torch.cuda.synchronize()
    a, b = out[..., rot:], q[..., rot:]
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(b)], b[~torch.isnan(b)])
    assert bool(torch.isfinite(out[..., :rot]).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_prepare_without_positions(R, interleaved):
    """Where nothing turns and no coordinates are kept, positions may be NULL."""
    n = 33
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(n, 6, 64, generator=g, device="cuda").half()
    q, km, vm = torch.empty(n, 4, 64, dtype=torch.float16, device="cuda"), *(torch.empty(n, 1, 64, dtype=torch.float16,
                                                                                         device="cuda") for _ in range(2))
    st = (6 * 64, 64)
    cfg = R.prepare_config(4, 1, 64, R.FP16, n, n, st, st, st, (256, 64), (64, 64), (64, 64), (0, 0, 0), interleaved=interleaved)
    R.check(R.rtcc_qkv_prepare(cfg, x.data_ptr(), x[:, 4:].data_ptr(), x[:, 5:].data_ptr(), None, None, None, None, q.data_ptr(),
                               km.data_ptr(), vm.data_ptr(), None))
    torch.cuda.synchronize()
    y = x.double() / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + 1e-6)
    for got, want in ((q, y[:, :4]), (km, y[:, 4:5])):
        assert bool(((got.double() - want).abs() <= (2.0 ** -11 + 2.0 ** -19) * want.abs() + 2.0 ** -25).all())
    assert torch.equal(vm, x[:, 5:])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def attend(R, q, k, v, n=None, m=None, dtype="fp16", begin=None, prefix=None, workspace=0, lse=True, out=None, **kw):
    """One call over whole tensors [rows][heads][dim]; `n` and `m` are the sequences'
    tokens and keys (default: one sequence of everything).  Returns (out, lse)."""
    n, m = [q.shape[0]] if n is None else n, [k.shape[0]] if m is None else m
    off, b = i32(np.concatenate([[0], np.cumsum(n)])), i32(np.concatenate([[0], np.cumsum(m)[:-1]]) if begin is None else begin)
    e = b + i32(m)
    p = None if prefix is None else i32(prefix)
    out = torch.full_like(q, 7.0) if out is None else out
    ls = torch.full(q.shape[:2], 7.0, device="cuda")
    ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    cfg = R.attn_config(q.shape[1], k.shape[1], q.shape[2], R.BF16 if dtype == "bf16" else R.FP16, q.shape[0], k.shape[0],
                        q.stride()[:2], k.stride()[:2], v.stride()[:2], out.stride()[:2], len(n), max(n), max(m), **kw)
    R.check(R.rtcc_memory_attention(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), off.data_ptr(), b.data_ptr(),
                                    e.data_ptr(), None if p is None else p.data_ptr(), None, None, None, None,
                                    out.data_ptr(), ls.data_ptr() if lse else None, ws.data_ptr() if workspace else None,
                                    workspace, 0))
    torch.cuda.synchronize()
    return out, ls


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("n,heads,lg,workspace", [(200, 1, 20, 64 << 20), (40, 2, 19, 64 << 20), (40, 1, 22, 0), (1, 1, 22, 1 << 20),
                                                  (2, 8, 20, 0), (1, 160, 20, 64 << 20)])
def test_attention_sums_over_many_equal_keys(R, n, heads, lg, workspace, dtype):
    """Equal scores over 2^19 to 2^22 keys.  The sums lose at most a unit in the last
    place per 16 keys: 2^-12 of a part of 65,536 keys, besides the usual 2 u + 2^-20."""
    m, dt = 1 << lg, torch.float16 if dtype == "fp16" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(lg)
    k = torch.zeros(m, heads, 8, device="cuda", dtype=dt)
    v = torch.rand(m, heads, 8, generator=g, device="cuda").to(dt)
    q = torch.zeros(n, heads, 8, device="cuda", dtype=dt)
    out, lse = attend(R, q, k, v, dtype=dtype, workspace=workspace)
    want = v.double().mean(0)
    u = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    err = (out.double() - want).abs() / want
    assert float(err.max()) <= 2 * u + 2.0 ** -12 + 2.0 ** -20
    assert float((lse.double() - lg * math.log(2)).abs().max()) <= 2.0 ** -20 * (1 + lg)


@pytest.mark.parametrize("n,workspace", [(1, 0), (1, 1 << 20), (3, 1 << 20), (40, 0), (40, 32 << 20), (200, 32 << 20)])
def test_attention_spans_up_to_the_limit(R, n, workspace):
    """2^31 - 2^16 equal keys and values: out is the value, lse the visible keys' logarithm (causal).
    Few rows read one row over and over (strides of 0); many need the rows themselves."""
    m = 2 ** 31 - 2 ** 16
    k = torch.full((1 if n <= 32 else m, 1, 8), 0.5, device="cuda", dtype=torch.float16)
    k = k.expand(m, 1, 8)
    q = torch.zeros(n, 1, 8, device="cuda", dtype=torch.float16)
    out, lse = attend(R, q, k, k, workspace=workspace, causal=True)
    assert bool((out == 0.5).all())
    want = torch.log(torch.arange(m - n + 1, m + 1, device="cuda", dtype=torch.float64))
    assert float((lse[:, 0].double() - want).abs().max()) <= 2.0 ** -20 * 23


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("m", [40, 300])
@pytest.mark.parametrize("dist", [False, True])
def test_attention_nan_stays_nan_under_a_cap(R, n, m, dist):
    """A NaN in a query makes its row NaN, and one in a key every row of its head, also where scores are
    capped; other rows keep their bits."""
    ref = Case([n, 5], [m, 300], heads=2, kv=2, cap=30.0, dist=dist).run(R).check()
    c = Case([n, 5], [m, 300], heads=2, kv=2, cap=30.0, dist=dist)
    c.q[0, 0, 3] = float("nan")
    c.k[m // 2, 1, 7] = float("nan")                 # of the first sequence
    c.run(R)
    torch.cuda.synchronize()
    bad = torch.zeros(n + 5, 2, dtype=torch.bool, device="cuda")
    bad[0, 0] = True
    bad[:n, 1] = True
    assert bool(torch.isnan(c.out[bad]).all()) and bool(torch.isnan(c.lse[bad]).all())
    assert torch.equal(c.out[~bad], ref.out[~bad]) and torch.equal(c.lse[~bad], ref.lse[~bad])


@pytest.mark.parametrize("n", [1, 200])
def test_attention_infinite_scores_reach_the_cap(R, n):
    """Scores of +-infinity are the cap and its negative."""
    q = torch.zeros(n, 1, 64, device="cuda", dtype=torch.bfloat16)
    k = torch.zeros(130, 1, 64, device="cuda", dtype=torch.bfloat16)
    q[:, 0, 0], k[7, 0, 0], k[100, 0, 0] = 3e38, 3e38, -3e38
    v = torch.zeros_like(k)
    v[7] = 1
    out, lse = attend(R, q, k, v, dtype="bf16", scale=1.0, cap=3.0)
    total = 128 + math.exp(3) + math.exp(-3)
    assert float((out.double() - math.exp(3) / total).abs().max()) <= 2 * 2.0 ** -8 * math.exp(3) / total
    assert float((lse.double() - math.log(total)).abs().max()) <= 4e-7 * 3 + 2.0 ** -20 * (1 + math.log(total))


@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("dist", [False, True])
@pytest.mark.parametrize("scale,sq,sk,dtype", [
    (1e-4, 150, 4, "fp16"), (1e-5, 150, 100, "fp16"), (1e-6, 500, 300, "fp16"), (1e-9, 1e4, 1e4, "bf16"),
    (1e-19, 1e9, 1e9, "bf16"), (-0.3, 3, 3, "fp16"), (-1e-5, 150, 100, "fp16")])
def test_attention_scales_and_caps(R, n, dist, scale, sq, sk, dtype):
    """Capped scores of up to 0.45 of the cap from queries and keys of any size, with scales down to 1e-19."""
    c = Case([n], [700], heads=2, kv=1, cap=30.0, dtype=dtype, dim=8, dist=dist)
    a = 0.45 * c.cap / (8 * abs(scale) * sq * sk)
    c.q.copy_(torch.sign(c.q) * sq * a)
    c.k.copy_(torch.sign(c.k) * sk)
    c.scale = scale
    c.run(R).check()


@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("scale,cap", [(-0.2, 0.0), (0.0, 0.0), (0.0, 20.0), (2.0, 1e-4), (30.0, 1e-4), (0.1, 1e-8)])
def test_attention_scales_of_any_sign_and_size(R, n, scale, cap):
    for dist in (False, True):
        c = Case([n, 3], [700, 90], heads=2, kv=1, cap=cap, dist=dist)
        c.scale = scale
        if scale < 0:                                # the check's score size is a magnitude
            c.q.neg_()
            ref = Case([n, 3], [700, 90], heads=2, kv=1, cap=cap, dist=dist)
            ref.scale = -scale
            c.run(R)
            ref.run(R).check()
            assert torch.equal(c.out, ref.out) and torch.equal(c.lse, ref.lse)
        else:
            c.run(R).check()


@pytest.mark.parametrize("n", [2, 200])
@pytest.mark.parametrize("cap", [300.0, 1e4, 1e5, 1e6, 1e30])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_large_caps_keep_relative_scores(R, n, cap, dtype):
    """Far above the scores a cap does next to nothing.  A capped score's error is 2^-20 of itself (tanh) and
    three roundings of 2^-24, besides the product's (float32 sums of 64 terms); no part of the cap."""
    c = Case([n], [700], heads=2, kv=1, cap=cap, dtype=dtype, spread=8.0).run(R)
    torch.cuda.synchronize()
    u = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    for h in range(2):
        q, k, v = c.q[:, h].double(), c.k[:, 0].double(), c.v[:, 0].double()
        x = cap * torch.tanh(c.scale * (q @ k.T) / cap)
        lse = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, None])
        size = c.scale * float((q.abs() @ k.abs().T).max())
        d = 2.0 ** -23 * 8 * size + (2.0 ** -20 + 3 * 2.0 ** -24) * float(x.abs().max()) + 2.0 ** -21
        err = (c.out[:, h].double() - p @ v).abs()
        assert bool((err <= (2 * u + 2 * d + 2.0 ** -20) * (p @ v.abs())).all())
        assert bool(((c.lse[:, h].double() - lse).abs() <= d + 2.0 ** -20 * (1 + lse.abs())).all())


@pytest.mark.parametrize("dim", [8, 72])
@pytest.mark.parametrize("heads,n,cap", [(160, 1, 0.0), (1, 200, 0.0), (1, 200, 1e6)])
def test_attention_sums_keep_small_probabilities(R, heads, n, cap, dim):
    """262,143 keys 2^-25 below the first one in the sum of their exponentials.  A warp (of four, few rows)
    or a row (many) adds n keys to one float32 sum: n 2^-28 of it may go, besides the usual 2^-20."""
    m = 1 << 18
    q = torch.zeros(n, heads, dim, device="cuda", dtype=torch.bfloat16)
    k = torch.zeros(m, heads, dim, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0], k[0, :, 0] = 1, 25
    _, lse = attend(R, q, k, k, dtype="bf16", scale=math.log(2), cap=cap)
    want = 25 * math.log(2) + math.log1p((m - 1) * 2.0 ** -25)
    lim = m * 2.0 ** -28 / (4 if n == 1 else 1) + 2.0 ** -20 * (1 + want) + 25 * 2.0 ** -20 + 2.0 ** -21
    assert float((lse.double() - want).abs().max()) <= lim


@pytest.mark.parametrize("heads,n", [(160, 1), (1, 200)])
@pytest.mark.parametrize("depth", [24.6, 25.1, 30.0])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_attention_long_tails_count(R, heads, n, depth, dtype):
    """One key far above 281,599 others, which together hold up to 1 % of the weight.  fp16 may lose 2^-40
    (few rows) or 2^-30 (many) of the largest probability per key, and a float32 sum over n keys (all of them,
    or a warp's quarter) n 2^-28 of itself."""
    m, dt = 281600, torch.float16 if dtype == "fp16" else torch.bfloat16
    q = torch.zeros(n, heads, 8, device="cuda", dtype=dt)
    q[:, :, :2] = 1
    u = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    for near in (0, 150000, m - 1):
        k = torch.zeros(m, heads, 8, device="cuda", dtype=dt)
        k[near, :, 0], k[near, :, 1] = math.floor(depth), depth - math.floor(depth)
        x = float(k[near, 0, :2].double().sum())
        v = torch.full_like(k, -1.0)
        v[near] = 1
        out, lse = attend(R, q, k, v, dtype=dtype, scale=math.log(2))
        rest = (m - 1) * 2.0 ** -x
        d = 2.0 ** -23 * math.sqrt(8) * x + 2.0 ** -21
        lost = 0 if dtype == "bf16" else m * (2.0 ** -40 if n == 1 else 2.0 ** -30)
        sums = m * 2.0 ** -28 / (4 if n == 1 else 1)
        assert float((out.double() - (1 - rest) / (1 + rest)).abs().max()) <= 2 * u + 2 * d + 2.0 ** -20 + lost + 2 * sums
        want = x * math.log(2) + math.log1p(rest)
        assert float((lse.double() - want).abs().max()) <= d + 2.0 ** -20 * (1 + want) + sums


def test_attention_rounds_each_probability_once(R):
    """A row whose maximum rises within a masked-form step, after the step's first 32 probabilities were
    rounded: 32 keys at 2^7.04, one at 2^8.03, the others, met before, at 1.  (Row 5's scores are twice as
    large, which makes its warp take that form.)  These values round up by 0.9 u again if scaled by 2^-8.03."""
    n, u = 200, 2.0 ** -8
    q = torch.zeros(n, 1, 64, device="cuda", dtype=torch.bfloat16)
    q[:, 0, :2] = 1
    q[5, 0, :2] = 2
    k = torch.zeros(128, 1, 64, device="cuda", dtype=torch.bfloat16)
    k[:32, 0, 0], k[:32, 0, 1] = 7, 10 / 256
    k[32, 0, 0], k[32, 0, 1] = 8, 7 / 256
    d = 2.0 ** -23 * 8 * 16 + 2.0 ** -21
    for j in range(128):
        v = torch.full_like(k, 1 + j / 128)
        out, _ = attend(R, q, k, v, dtype="bf16", scale=math.log(2))
        assert float((out.double() / (1 + j / 128) - 1).abs().max()) <= 2 * u + 2 * d + 2.0 ** -20, j


def check_causal(out, lse, q, k, v, n, m, begin, start, prefix, u):
    """float64 attention with key j of a sequence visible to its token i where j <= start + i or j < prefix."""
    at, group = 0, q.shape[1] // k.shape[1]
    for s in range(len(n)):
        i, j = torch.arange(n[s], device="cuda")[:, None], torch.arange(m[s], device="cuda")[None]
        see = (j <= i + start[s]) | (j < prefix[s])
        for h in range(q.shape[1]):
            kk, vv = k[begin[s]:begin[s] + m[s], h // group].double(), v[begin[s]:begin[s] + m[s], h // group].double()
            some = see.any(0)[:, None]
            kk, vv = torch.where(some, kk, 0.0), torch.where(some, vv, 0.0)
            qq = q[at:at + n[s], h].double()
            x = torch.where(see, qq @ kk.T / math.sqrt(q.shape[2]), -math.inf)
            want_lse = torch.logsumexp(x, 1) if m[s] else torch.full((n[s],), -math.inf, device="cuda", dtype=torch.float64)
            none = torch.isinf(want_lse)
            p = torch.exp(x - torch.where(none, 0.0, want_lse)[:, None])
            size = float((qq.abs() @ kk.abs().T).max()) / math.sqrt(q.shape[2]) if n[s] and m[s] else 0.0
            d = 2.0 ** -23 * math.sqrt(q.shape[2]) * size + 2.0 ** -21
            err = (out[at:at + n[s], h].double() - p @ vv).abs()
            assert bool((err <= (2 * u + 2 * d + 2.0 ** -20) * (p @ vv.abs()) + 2.0 ** -25).all()), (s, h)
            got = lse[at:at + n[s], h].double()
            assert bool((got[none] == -math.inf).all())
            assert bool(((got - want_lse).abs()[~none] <= d + 2.0 ** -20 * (1 + want_lse[~none].abs())).all()), (s, h)
        at += n[s]


@pytest.mark.parametrize("n,m", [([4, 1, 3], [12, 40, 3]), ([30, 200], [64, 130]), ([150, 0, 300], [400, 10, 90])])
@pytest.mark.parametrize("kind", ["held", "behind", "ahead"])
@pytest.mark.parametrize("prefixed", [False, True])
def test_attention_starts(R, n, m, kind, prefixed):
    """Starts at any place among the keys; keys that no token sees then hold NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(len(n) + n[0])
    start = {"held": [max(0, b - a + 2) for a, b in zip(n, m)], "behind": [max(0, b - a - 37) // 2 for a, b in zip(n, m)],
             "ahead": [b + 10 for b in m]}[kind]
    prefix = [min(b, 29) for b in m] if prefixed else [0] * len(m)
    q = torch.randn(sum(n), 4, 64, generator=g, device="cuda").half()
    k = torch.randn(sum(m), 2, 64, generator=g, device="cuda").half()
    v = torch.randn(sum(m), 2, 64, generator=g, device="cuda").half()
    begin = np.concatenate([[0], np.cumsum(m)[:-1]]).tolist()
    for a, b, s, p, at in zip(n, m, start, prefix, begin):
        seen = min(b, max(p, s + a))
        k[at + seen:at + b], v[at + seen:at + b] = float("nan"), float("inf")
    st = i32(start)
    for workspace in (0, 16 << 20):
        out, lse = attend(R, q, k, v, n=n, m=m, prefix=prefix if prefixed else None, workspace=workspace, causal=True,
                          q_start=st.data_ptr())
        check_causal(out, lse, q, k, v, n, m, begin, start, prefix, 2.0 ** -11)


def test_attention_negative_starts_read_as_zero(R):
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    for n, m in (([3], [9]), ([150], [400])):
        q = torch.randn(n[0], 2, 64, generator=g, device="cuda").half()
        k, v = (torch.randn(m[0], 2, 64, generator=g, device="cuda").half() for _ in range(2))
        st = i32([-5])
        out, lse = attend(R, q, k, v, causal=True, q_start=st.data_ptr())
        check_causal(out, lse, q, k, v, n, m, [0], [0], [0], 2.0 ** -11)


@pytest.mark.parametrize("n_new", [[4, 3, 0], [60, 2, 90]])
def test_append_into_slots_that_fill_up_then_attend(R, n_new):
    """Tokens that still got a row see it and what came before it; those past the capacity see the slot."""
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(n_new))
    seqs, capacity, held_h = 3, 80, [78, 20, 10]
    n = sum(n_new)
    e = lambda c: torch.empty(c, dtype=torch.int32, device="cuda")  # noqa: E731
    off, rows, begin, end, length = e(seqs + 1), e(n), e(seqs), e(seqs), e(seqs)
    held, fresh = i32(held_h), i32(n_new)
    R.check(R.rtcc_memory_append(seqs, capacity, n, fresh.data_ptr(), held.data_ptr(), None, off.data_ptr(), rows.data_ptr(),
                                 None, None, begin.data_ptr(), end.data_ptr(), length.data_ptr()))
    k = torch.randn(seqs * capacity, 2, 64, generator=g, device="cuda").half()
    v = torch.randn(seqs * capacity, 2, 64, generator=g, device="cuda").half()
    q = torch.randn(n, 2, 64, generator=g, device="cuda").half()
    out, lse = torch.empty_like(q), torch.empty(n, 2, device="cuda")
    st = (128, 64)
    cfg = R.attn_config(2, 2, 64, R.FP16, n, seqs * capacity, st, st, st, st, seqs, max(n_new), capacity, causal=True,
                        q_start=held.data_ptr())
    R.check(R.rtcc_memory_attention(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), off.data_ptr(), begin.data_ptr(),
                                    end.data_ptr(), None, None, None, None, None, out.data_ptr(), lse.data_ptr(), None, 0))
    torch.cuda.synchronize()
    m = [min(capacity, h + a) for h, a in zip(held_h, n_new)]
    assert length.tolist() == m
    check_causal(out, lse, q, k, v, n_new, m, [s * capacity for s in range(seqs)], held_h, [0] * seqs, 2.0 ** -11)


@pytest.mark.parametrize("max_q", [40, 129, 200])
@pytest.mark.parametrize("n,m", [([400], [1000]), ([700, 0, 333], [777, 64, 1500]), ([1500], [700]), ([401, 399], [0, 2177])])
@pytest.mark.parametrize("kw", [
    dict(heads=2, kv=2, dim=64), dict(heads=3, kv=1, dim=128, causal=True, prefixed=90, dtype="bf16"),
    dict(heads=2, kv=1, dim=64, cap=20.0, dist=True), dict(heads=4, kv=2, dim=128, slot_rows=150, absent=(0, 2, 3), cap=30.0),
    dict(heads=1, kv=1, dim=80, causal=True, dist=True, slot_rows=100, absent=(1, 4), dtype="bf16")])
def test_attention_longer_sequences_than_stated(R, max_q, n, m, kw):
    """The blocks of the many-rows kernel then take several groups of rows, one after another: with one or two
    streams, other groups' masks, steps and ring places."""
    kw = dict(kw)
    if kw.get("absent"):
        kw["absent"] = [a for a in kw["absent"] if a * kw["slot_rows"] < sum(m) + 7 * (len(m) + 1)]
    prefix = kw.pop("prefixed", None)
    c = Case(n, m, gap=7, prefix=None if prefix is None else [min(prefix, x) for x in m], seed=max_q, **kw)
    for run in (dict(workspace=0), dict(), dict(max_k=300), dict(workspace=0, max_k=64)):
        c.out.fill_(7.0)
        c.run(R, max_q=max_q, **run).check()
    assert R.rtcc_memory_attention_status() == R.OK


# ---------------------------------------------------------------------------
# waits and launches that fail
# ---------------------------------------------------------------------------

@pytest.fixture
def hook(R):
    yield R.rtcc_test_attention
    R.rtcc_test_attention(0)


@pytest.mark.parametrize("kw", [
    dict(n=[300], m=[500], heads=2, kv=2), dict(n=[40, 200], m=[5000, 130], heads=4, kv=2, dim=128, causal=True, dtype="bf16"),
    dict(n=[200], m=[20000], heads=1, kv=1, cap=20.0, dist=True, slot_rows=1000, absent=(3, 7)), dict(n=[256], m=[64], heads=1, kv=1)])
def test_attention_wait_that_runs_out_is_reported(R, hook, kw):
    """A kernel whose queries never come gives its waits up; the report says so once, and the calls before and
    after are right."""
    assert R.rtcc_memory_attention_status() == R.OK
    c = Case(**kw).run(R).check()
    assert R.rtcc_memory_attention_status() == R.OK
    first = c.out.clone()
    assert hook(R.TEST_UNREACHABLE_WAIT) == R.OK
    c.run(R)
    assert R.rtcc_memory_attention_status() == R.E_DEVICE
    assert hook(0) == R.OK
    assert R.rtcc_memory_attention_status() == R.OK
    c.out.fill_(7.0)
    c.run(R).check()
    assert torch.equal(c.out, first) and R.rtcc_memory_attention_status() == R.OK


def test_attention_failure_is_reported_to_every_stream(R, hook):
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    R.rtcc_memory_attention_status(a.cuda_stream), R.rtcc_memory_attention_status(b.cuda_stream)
    c = Case([300], [500], heads=2, kv=2)
    torch.cuda.synchronize()
    hook(R.TEST_UNREACHABLE_WAIT)
    with torch.cuda.stream(a):
        c.run(R, stream=a.cuda_stream)
    a.synchronize()
    hook(0)
    # the report on b does not take a's away
    assert R.rtcc_memory_attention_status(b.cuda_stream) == R.E_DEVICE
    assert R.rtcc_memory_attention_status(a.cuda_stream) == R.E_DEVICE
    assert R.rtcc_memory_attention_status(a.cuda_stream) == R.OK
    assert R.rtcc_memory_attention_status(b.cuda_stream) == R.OK
    assert R.rtcc_memory_attention_status() == R.E_DEVICE
    assert R.rtcc_memory_attention_status() == R.OK


@pytest.mark.parametrize("workspace", [0, 32 << 20])
def test_attention_without_clusters(R, hook, workspace):
    """A refused cluster launch is made up for by split spans, and with no workspace by whole ones."""
    for n, m, dim in (([1], [4097], 64), ([2, 0, 4, 1], [1, 700, 2000, 650], 80), ([3], [2049], 128)):
        c = Case(n, m, heads=6, kv=2, dim=dim, causal=True)
        hook(R.TEST_NO_CLUSTERS)
        c.run(R, workspace=workspace).check()
        hook(0)
        c.out.fill_(7.0)
        c.run(R, workspace=workspace).check()
