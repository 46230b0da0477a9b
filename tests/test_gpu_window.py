"""Attention with a sliding window and sinks on the GPU against the plain float64
form; tolerances as in test_gpu_tokens.py.  Rows that no token sees hold NaN."""
import math

import numpy as np
import pytest

from tests import gpu_util as U
from tests.test_gpu_tokens import Case, i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def R():
    return U.load()


class Window(Case):
    def __init__(self, n, m, window, sinks=0, start=None, **kw):
        super().__init__(n, m, causal=True, **kw)
        self.window, self.sinks = window, sinks
        self.start = [b - a for a, b in zip(self.n, self.m)] if start is None else list(start)
        self.given = start is not None
        hidden = torch.ones(self.rows, dtype=torch.bool, device="cuda")
        for s in range(len(self.n)):
            see = torch.tensor(self.visible(s).any(0), device="cuda")
            hidden[self.begin[s]:self.begin[s] + self.m[s]] &= ~see
        self.k[hidden] = float("nan")
        self.v[hidden] = float("inf")
        if self.k_pos is not None:
            self.k_pos[hidden] = float("nan")

    def visible(self, s):
        n, m, b = self.n[s], self.m[s], self.begin[s]
        if not hasattr(self, "window"):
            return np.ones((n, m), dtype=bool)
        p, j = np.arange(n)[:, None] + self.start[s], np.arange(m)[None]
        see = (j <= p) & ((j > p - self.window) | (j < self.sinks))
        if self.prefix is not None:
            see = see | (j < self.prefix[s])
        if self.slot_rows:
            see = see & (self.present.cpu().numpy()[(b + np.arange(m)) // self.slot_rows] != 0)[None]
        return see

    def run(self, R, workspace=32 << 20, max_q=None, max_k=None, stream=0):
        p = lambda t: None if t is None or not t.numel() else t.data_ptr()  # noqa: E731
        self.off_d = i32(np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32))
        self.b_d, self.e_d = i32(self.begin), i32([b + x for b, x in zip(self.begin, self.m)])
        self.p_d = None if self.prefix is None else i32(self.prefix)
        self.s_d = i32(self.start) if self.given else None
        self.ws = torch.full((max(workspace, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        self.cfg = R.attn_config(self.heads, self.kv, self.dim, R.BF16 if self.dtype == "bf16" else R.FP16, self.tokens,
                                 self.rows, self.q.stride()[:2], self.k.stride()[:2], self.v.stride()[:2],
                                 self.out.stride()[:2], len(self.n), max(self.n + [0]) if max_q is None else max_q,
                                 max(self.m + [0]) if max_k is None else max_k, causal=True,
                                 n_slots=0 if self.present is None else self.present.numel(), slot_rows=self.slot_rows,
                                 q_pos_row=3, scale=self.scale, cap=self.cap, q_start=p(self.s_d))
        self.args = [self.cfg, self.window, self.sinks, p(self.q), p(self.k), p(self.v), p(self.off_d), p(self.b_d),
                     p(self.e_d), p(self.p_d), p(self.present), p(self.slopes), p(self.q_pos), p(self.k_pos), p(self.out),
                     p(self.lse), self.ws.data_ptr() if workspace else None, workspace]
        R.check(R.rtcc_memory_window_attention(*self.args, stream))
        return self


SHAPES = [
    # tokens, keys, window, sinks
    ([1], [1], 1, 0), ([1], [500], 1, 0), ([1], [500], 100, 3), ([1], [5000], 700, 16), ([1], [5000], 9000, 4),
    ([1], [129], 64, 64), ([1], [4096], 64, 1), ([3], [1000], 50, 70), ([17], [1000], 5, 0), ([40], [3000], 333, 130),
    ([100], [100], 1, 0), ([130], [130], 7, 200), ([200], [5000], 640, 64), ([300], [300], 64, 0), ([500], [2000], 1, 1),
    ([700], [700], 100, 10), ([257], [10000], 2000, 65), ([1, 1, 1, 1], [1, 0, 777, 4096], 300, 5),
    ([0, 3, 0, 40], [10, 3, 0, 200], 20, 2), ([5, 64, 200, 1], [0, 64, 333, 1], 30, 9), ([30], [20], 4, 3),
    ([300, 129], [290, 5000], 128, 128),
]


@pytest.mark.parametrize("n,m,window,sinks", SHAPES)
@pytest.mark.parametrize("dim,heads,kv,dtype", [(64, 2, 2, "fp16"), (128, 4, 1, "bf16")])
def test_window_lengths(R, n, m, window, sinks, dim, heads, kv, dtype):
    Window(n, m, window, sinks, dim=dim, heads=heads, kv=kv, dtype=dtype, gap=3).run(R).check()


@pytest.mark.parametrize("n,m", [(1, 3000), (9, 700), (150, 1300)])
@pytest.mark.parametrize("dim,dtype", [(8, "fp16"), (40, "bf16"), (80, "fp16"), (104, "bf16")])
def test_window_head_sizes(R, n, m, dim, dtype):
    Window([n, n], [m, m - 5], 200, 20, dim=dim, heads=3, kv=1, dtype=dtype).run(R).check()


@pytest.mark.parametrize("n,m,dim", [(1, 3000, 64), (9, 700, 128), (150, 1300, 64), (260, 900, 128)])
@pytest.mark.parametrize("cap,dist", [(0.0, True), (20.0, False), (20.0, True), (500.0, False)])
def test_window_scores(R, n, m, dim, cap, dist):
    Window([n, n // 2 + 1], [m, m // 2 + 40], 170, 6, dim=dim, heads=2, kv=2, cap=cap, dist=dist, spread=3).run(R).check()


@pytest.mark.parametrize("n,m", [(1, 3000), (20, 1000), (150, 1300), (400, 400)])
def test_window_with_a_prefix(R, n, m):
    """A prefix all tokens see, later ones too; longer than the window, and none."""
    for prefix in ([0, 7], [m, 1], [100, 333]):
        Window([n, n], [m, m], 64, 5, heads=4, kv=2, dim=64, prefix=prefix).run(R).check()


@pytest.mark.parametrize("slot_rows,absent,n", [(100, (1, 4), 1), (100, (0,), 40), (64, (2, 3, 5), 200), (77, (1, 2, 6), 300)])
def test_window_absent_slots(R, slot_rows, absent, n):
    Window([n], [900], 400, 150, heads=2, kv=2, slot_rows=slot_rows, absent=absent).run(R).check()
    Window([n], [900], 30, 2, heads=2, kv=2, slot_rows=slot_rows, absent=absent, dist=True).run(R).check()


@pytest.mark.parametrize("n", [1, 8, 200])
def test_window_given_starts(R, n):
    """Tokens that got no key (a full slot), and keys after the last token's."""
    m = 1000
    Window([n, n, n], [m, m, m], 90, 4, start=[m - n, m - n // 2, 100], heads=2, kv=1, dim=64).run(R).check()
    Window([n], [m], 50, 0, start=[m], heads=2, kv=1, dim=64).run(R).check()


@pytest.mark.parametrize("n,m,window", [(1, 60000, 40000), (2, 9000, 8000), (40, 9000, 3000), (300, 9000, 5000)])
def test_window_split_and_hints(R, n, m, window):
    """Any split, none, and wrong hints of the lengths give the same result."""
    for kw in (dict(), dict(workspace=0), dict(workspace=200000), dict(max_q=1, max_k=1), dict(max_q=9, max_k=70)):
        Window([n, 3], [m, 200], window, 33, heads=2, kv=1, dim=64).run(R, **kw).check()


def test_window_as_wide_as_the_span_is_plain_attention(R):
    for n, m in ((1, 3000), (30, 700), (300, 700)):
        a = Case([n], [m], heads=2, kv=1, causal=True).run(R).check()
        b = Window([n], [m], 1 << 30, 0, heads=2, kv=1).run(R)
        for window, sinks in ((2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1)):
            Window([n], [m], window, sinks, heads=2, kv=1).run(R).check()
        torch.cuda.synchronize()
        assert float((a.out.float() - b.out.float()).abs().max()) <= 2.0 ** -9


def test_window_repeats_in_a_graph_on_a_side_stream(R):
    for n, m in (([1, 1], [5000, 300]), ([40], [900]), ([300], [1900])):
        c = Window(n, m, 250, 3, heads=2, kv=1, dim=128)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        c.run(R, stream=s.cuda_stream)
        s.synchronize()
        c.check()
        first, lse = c.out.clone(), c.lse.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            R.check(R.rtcc_memory_window_attention(*c.args, torch.cuda.current_stream().cuda_stream))
        for _ in range(3):
            c.out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, first) and torch.equal(c.lse, lse)


def test_window_untouched_tokens_and_status(R):
    c = Window([5, 200], [300, 300], 40, 2, heads=2, kv=2)
    c.off = None
    c.run(R)
    off = i32([0, 5, 100])                                    # the rest belongs to no sequence
    c.out.fill_(7)
    c.args[6] = off.data_ptr()
    R.check(R.rtcc_memory_window_attention(*c.args, 0))
    torch.cuda.synchronize()
    assert (c.out[100:] == 7).all() and not (c.out[:100] == 7).all()
    assert R.rtcc_memory_attention_status() == R.OK


# sizes that the tensor-core kernel takes: more than 32 rows of a key head, and more than
# 200,000 pairs of a block of 16 of them and a key
LARGE = [([1500], [1500], 100, 10), ([700, 900], [2700, 900], 640, 64), ([1300], [5000], 1, 0), ([1025], [1025], 1024, 0),
         ([600, 1, 0, 65], [4096, 900, 10, 3000], 1777, 130), ([900], [890], 64, 63), ([1100], [1100], 63, 65)]


@pytest.mark.parametrize("n,m,window,sinks", LARGE)
@pytest.mark.parametrize("dim,heads,kv,dtype", [(64, 2, 2, "fp16"), (128, 4, 2, "bf16"), (72, 3, 3, "bf16")])
def test_window_large(R, n, m, window, sinks, dim, heads, kv, dtype):
    Window(n, m, window, sinks, dim=dim, heads=heads, kv=kv, dtype=dtype, gap=3).run(R).check()


@pytest.mark.parametrize("cap,dist,dim", [(0.0, True, 64), (20.0, False, 128), (20.0, True, 64), (500.0, False, 64)])
def test_window_large_scores(R, cap, dist, dim):
    Window([1000, 333], [1300, 2000], 170, 6, dim=dim, heads=4, kv=4, cap=cap, dist=dist, spread=3).run(R).check()


def test_window_large_with_prefix_starts_and_slots(R):
    Window([1100, 900], [1100, 2000], 64, 5, heads=4, kv=2, prefix=[100, 777]).run(R).check()
    Window([1100, 900], [1100, 2000], 64, 5, heads=4, kv=2, start=[600, 1300]).run(R).check()
    for window, sinks in ((400, 150), (30, 2)):
        Window([1200], [2400], window, sinks, heads=4, kv=4, slot_rows=100, absent=(0, 1, 7, 13, 14)).run(R).check()
        Window([1200], [2400], window, sinks, heads=2, kv=2, slot_rows=77, absent=(2, 20), dist=True).run(R).check()


def test_window_large_split_and_hints(R):
    """Long windows split over the GPU with room for parts, one tile at a time, and wrong hints."""
    for kw in (dict(), dict(workspace=0), dict(workspace=16 << 20), dict(max_q=40, max_k=4000)):
        Window([300], [9000], 7000, 33, heads=4, kv=2, dim=64).run(R, **kw).check()
        Window([100], [9000], 8000, 33, heads=3, kv=3, dim=128).run(R, **kw).check()


def test_window_large_repeats_and_keeps_bits(R):
    a = Window([1300], [1300], 200, 9, heads=4, kv=2, dim=128).run(R)
    b = Window([1300], [1300], 200, 9, heads=4, kv=2, dim=128).run(R)
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


def test_window_given_up_wait_is_reported(R):
    """The queries never come: every wait ends by itself, the status tells, and the next call is right."""
    assert R.rtcc_memory_attention_status() == R.OK
    c = Window([1300], [1300], 200, 9, heads=4, kv=2)
    try:
        assert R.rtcc_test_attention(R.TEST_UNREACHABLE_WAIT) == R.OK
        c.run(R)
        assert R.rtcc_memory_attention_status() == R.E_DEVICE
    finally:
        assert R.rtcc_test_attention(0) == R.OK
    assert R.rtcc_memory_attention_status() == R.OK
    c.run(R).check()


def test_window_without_clusters(R):
    for workspace in (0, 32 << 20):
        try:
            assert R.rtcc_test_attention(R.TEST_NO_CLUSTERS) == R.OK
            c = Window([1], [4000], 3000, 9, heads=2, kv=2).run(R, workspace=workspace)
        finally:
            assert R.rtcc_test_attention(0) == R.OK
        c.check()


@pytest.mark.parametrize("n,m", [(1, 1000), (8, 1000), (200, 777), (1300, 1500)])
@pytest.mark.parametrize("dim,heads,kv,dtype", [(64, 4, 4, "fp16"), (128, 4, 2, "bf16")])
def test_window_starts_behind_the_span(R, n, m, dim, heads, kv, dtype):
    """Tokens at places past the last key: their windows reach back over fewer keys, or none."""
    for window, sinks in ((50, 0), (50, 7), (640, 64), (3000, 0)):
        for start in ([m, m + 30, m + 1], [m + 100, m - n, m + 700], [2 ** 31 - 1, m + window, m + window - 1]):
            Window([n, n, 2], [m, m, m], window, sinks, start=start, dim=dim, heads=heads, kv=kv, dtype=dtype).run(R).check()
    Window([n, n], [m, m], 50, 3, start=[m + 500, 2 ** 31 - 1], prefix=[0, 300], dim=dim, heads=heads, kv=kv, dtype=dtype).run(R).check()


@pytest.mark.parametrize("pages", [False, True])
@pytest.mark.parametrize("n,window,seen", [(200, 64, 700001), (200, 150, 1000000), (70, 64, 700001)])
@pytest.mark.parametrize("by", ["prefix", "sinks"])
def test_window_behind_a_long_shared_part(R, pages, n, window, seen, by):
    """More tokens than a window is long, all of which see the same long part: sums over no
    more than 65,536 keys of equal weight there too.  The tensor cores add four keys' products to
    a sum at a time and cut it by a unit in the last place at most.  A sum that ends in
    [2^k, 2^(k + 1)) at S = t 2^k over N keys was in that octave for (1 - 1/t) N keys, N (1 - 1/t) / 4
    units of 2^(k - 23), and below for N / t, which cost N / (6 t) 2^(k - 24): together, over S,
    N 2^-24 (1/2 - 1/(3 t)) / t, largest at t = 4/3: 3/16 N 2^-24 = 3 N 2^-28, 3 2^-12 for 65,536 keys.  The
    result's rounding is 2^-11.  The shared keys weigh
    1365/1024 of the windows' (11 bits, so rounding them costs nothing) and all values are 15/8,
    so that 16 products add up to a number with fraction bits for the sum to lose."""
    m, heads, kv, dim = seen + 500, 2, 1, 64
    weight, value = 1365 / 1024, 1.875
    q = torch.zeros(n, heads, dim, device="cuda").half()
    q[..., 0] = 1
    out, lse = torch.zeros_like(q), torch.zeros(n, heads, device="cuda")
    off, end, ws = i32([0, n]), i32([m]), torch.full((192 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    prefix, sinks = (i32([seen]), 0) if by == "prefix" else (None, seen)
    pre, scale = None if prefix is None else prefix.data_ptr(), math.log(weight)
    per = -(-m // 128)
    k, v = torch.zeros(per * 128, kv, dim, device="cuda"), torch.full((per * 128, kv, dim), value, device="cuda")
    k[:seen, :, 0] = 1
    if pages:
        k, v = (t.view(per, 128, kv, dim).transpose(1, 2).contiguous().to(torch.float8_e4m3fn).view(torch.uint8) for t in (k, v))
        e, table = torch.zeros(per, kv, 8, 2, device="cuda", dtype=torch.int8), i32(list(range(per)))
        R.check(R.rtcc_pages_attention(
            R.page_config(kv, dim, 128, per, 1, per),
            R.page_attn_config(heads, R.FP16, n, q.stride()[:2], out.stride()[:2], n, m, window=window, sinks=sinks, scale=scale),
            q.data_ptr(), off.data_ptr(), None, end.data_ptr(), pre, table.data_ptr(), k.data_ptr(), v.data_ptr(), e.data_ptr(),
            out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel()))
    else:
        k, v, begin = k.half(), v.half(), i32([0])
        cfg = R.attn_config(heads, kv, dim, R.FP16, n, m, q.stride()[:2], k.stride()[:2], v.stride()[:2], out.stride()[:2], 1, n, m,
                            causal=True, scale=scale)
        R.check(R.rtcc_memory_window_attention(cfg, window, sinks, q.data_ptr(), k.data_ptr(), v.data_ptr(), off.data_ptr(),
                                               begin.data_ptr(), end.data_ptr(), pre, None, None, None, None, out.data_ptr(),
                                               lse.data_ptr(), ws.data_ptr(), ws.numel()))
    torch.cuda.synchronize()
    assert float((out.double() / value - 1).abs().max()) <= 2.0 ** -11 + 3 * 2.0 ** -12 + 2.0 ** -20
    assert float((lse.double() - math.log(seen * weight + window)).abs().max()) <= 2.0 ** -20 * 15


@pytest.mark.parametrize("window,sinks,cap,dist", [(200, 9, 0.0, False), (200, 9, 20.0, False), (200, 9, 0.0, True), (1, 0, 0.0, False)])
def test_window_non_finite_queries_stay_in_their_rows(R, window, sinks, cap, dist):
    for n, m in ((1500, 1500), (300, 9000), (6, 700)):
        make = lambda: Window([n], [m], window, sinks, heads=4, kv=4, dim=64, cap=cap, dist=dist)  # noqa: E731
        c, ref = make(), make().run(R).check()
        q, bad = c.q.clone(), [(0, 0), (n // 2, 1), (n - 1, 3), (n // 3, 2)]
        for i, (t, h) in enumerate(bad):
            c.q[t, h, 5 * i] = float("nan")
            c.q[t, h, 7] = float("inf")
        c.run(R)
        torch.cuda.synchronize()
        for t, h in bad:
            assert torch.isnan(c.out[t, h]).all() and torch.isnan(c.lse[t, h])
            c.out[t, h], c.lse[t, h] = ref.out[t, h], ref.lse[t, h]
        c.q.copy_(q)
        c.check()
