"""Paged token memory and windowed attention without a GPU: every refusal comes
before any GPU work, and empty calls succeed."""
import pytest

from paper_2608_08330_gb300 import build as B

P = 0x10000            # an aligned address; refused calls never read it


@pytest.fixture(scope="module")
def R():
    B.build()
    from paper_2608_08330_gb300 import rtcc
    rtcc.load()
    return rtcc


def cfg(R, **kw):
    a = dict(kv_heads=2, head_dim=64, page_rows=64, n_pages=10, n_seqs=3, table_row=4)
    a.update(kw)
    return R.page_config(**a)


BAD_SHAPES = (dict(kv_heads=0), dict(kv_heads=4097), dict(head_dim=0), dict(head_dim=8), dict(head_dim=72),
              dict(head_dim=144), dict(page_rows=0), dict(page_rows=16), dict(page_rows=48), dict(page_rows=256),
              dict(n_pages=-1), dict(n_pages=2 ** 26 + 1), dict(n_seqs=-1), dict(table_row=-1),
              dict(table_row=2 ** 24 + 1), dict(n_seqs=2 ** 16, table_row=2 ** 15), dict(page_bytes=8),
              dict(page_bytes=8200), dict(page_bytes=4096), dict(page_bytes=-16), dict(scale_bytes=2), dict(scale_bytes=12),
              dict(scale_bytes=18), dict(page_bytes=2 ** 41))


def fork(R, c, n_from=5, window=0, sinks=0, **kw):
    a = dict(parent=P, keep=None, length=P + 0x100, table=P + 0x200, length_out=P + 0x1000, table_out=P + 0x2000,
             refs=P + 0x3000)
    a.update(kw)
    return R.rtcc_pages_fork(c, n_from, a["parent"], a["keep"], window, sinks, a["length"], a["table"], a["length_out"],
                             a["table_out"], a["refs"])


def extend(R, c, nbytes=4096, **kw):
    a = dict(new=P, length=P + 0x100, table=P + 0x200, refs=P + 0x400, length_out=P + 0x500, src=P + 0x600, dst=P + 0x700,
             rows=P + 0x800, short=P + 0x900, workspace=P + 0x10000)
    a.update(kw)
    return R.rtcc_pages_extend(c, *a.values(), nbytes)


def compact(R, c, nbytes=4096, **kw):
    a = dict(table=P, refs=P + 0x200, table_out=P + 0x400, refs_out=P + 0x600, src=P + 0x700, dst=P + 0x800,
             count=P + 0x900, workspace=P + 0x10000)
    a.update(kw)
    return R.rtcc_pages_compact(c, *a.values(), nbytes)


def copy(R, c, n=3, n_dst=7, **kw):
    a = dict(count=None, src=P, dst=P, rows=None, k=P, v=P, s=P, k2=P, v2=P, s2=P)
    a.update(kw)
    v = list(a.values())
    return R.rtcc_pages_copy(c, n, *v[:7], n_dst, *v[7:])


def write(R, c, tokens=None, **kw):
    a = dict(k=P, v=P, offsets=P, held=P, length=None, table=P, k_pages=P, v_pages=P, scales=P)
    a.update(kw)
    return R.rtcc_pages_write(c, tokens or R.write_config(R.FP16, 5, 2, (128, 64), (128, 64)), *a.values())


def rows_cfg(R, **kw):
    a = dict(heads=4, dtype=R.FP16, n_q=5, q=(256, 64), out=(256, 64), max_q=2, max_k=100, scale=0.1)
    a.update(kw)
    return R.page_attn_config(**a)


def attend(R, c, rows, **kw):
    a = dict(q=P, offsets=P, start=None, length=P, prefix=None, table=P, k=P, v=P, s=P, out=P, lse=None, ws=None)
    a.update(kw)
    return R.rtcc_pages_attention(c, rows, *a.values(), 0)


def test_shapes_are_refused_by_every_call(R):
    for kw in BAD_SHAPES:
        c = cfg(R, **kw)
        assert R.rtcc_pages_workspace(c) == 0, kw
        assert fork(R, c) == R.E_ARG, kw
        assert extend(R, c) == R.E_ARG, kw
        assert compact(R, c) == R.E_ARG, kw
        assert copy(R, c) == R.E_ARG, kw
        assert write(R, c) == R.E_ARG, kw
        assert attend(R, c, rows_cfg(R)) == R.E_ARG, kw
    lib = R.load()
    assert lib.rtcc_pages_fork(None, 0, None, None, 0, 0, None, None, None, None, None, None) == R.E_ARG
    assert lib.rtcc_pages_write(cfg(R), None, *[None] * 10) == R.E_ARG
    assert R.rtcc_pages_workspace(cfg(R)) >= 4 * (10 + 3)


def test_fork_refusals(R):
    c = cfg(R)
    assert fork(R, c, n_from=-1) == R.E_ARG and fork(R, c, window=-1) == R.E_ARG and fork(R, c, sinks=-1) == R.E_ARG
    assert fork(R, c, n_from=2 ** 30) == R.E_ARG
    for name in ("parent", "length", "table", "length_out", "table_out", "refs"):
        assert fork(R, c, **{name: None}) == R.E_ARG, name
    for name in ("parent", "keep", "length", "table", "length_out", "table_out", "refs"):
        assert fork(R, c, **{name: P + 0x4002}) == R.E_ARG, name
    assert fork(R, c, table_out=P + 0x200) == R.E_ARG           # in place
    assert fork(R, c, table_out=P + 0x200 + 4 * 5 * 4 - 4) == R.E_ARG       # over the old table's end
    assert fork(R, c, length_out=P + 0x100) == R.E_ARG and fork(R, c, refs=P) == R.E_ARG
    assert fork(R, cfg(R, n_pages=0, n_seqs=0)) == R.OK


def test_extend_and_compact_refusals(R):
    c = cfg(R)
    for name in ("new", "length", "table", "refs", "length_out", "src", "dst", "rows", "workspace"):
        assert extend(R, c, **{name: None}) == R.E_ARG, name
        assert extend(R, c, **{name: P + 0x20002}) == R.E_ARG, name
    assert extend(R, c, short=P + 0x20002) == R.E_ARG
    assert extend(R, c, nbytes=R.rtcc_pages_workspace(c) - 1) == R.E_ARG
    assert extend(R, c, workspace=P + 0x10008) == R.E_ARG
    assert extend(R, c, src=P + 0x700) == R.E_ARG and extend(R, c, length_out=P) == R.E_ARG
    assert extend(R, c, workspace=P + 0x200) == R.E_ARG and extend(R, c, refs=P + 0x200) == R.E_ARG
    for name in ("table", "refs", "table_out", "refs_out", "src", "dst", "count", "workspace"):
        assert compact(R, c, **{name: None}) == R.E_ARG, name
        assert compact(R, c, **{name: P + 0x20002}) == R.E_ARG, name
    assert compact(R, c, nbytes=R.rtcc_pages_workspace(c) - 1) == R.E_ARG
    assert compact(R, c, refs_out=P + 0x200) == R.E_ARG and compact(R, c, src=P + 0x800) == R.E_ARG
    assert compact(R, c, table_out=P + 4) == R.E_ARG


def test_copy_refusals(R):
    c = cfg(R)
    assert copy(R, c, n=-1) == R.E_ARG and copy(R, c, n_dst=-1) == R.E_ARG and copy(R, c, n_dst=2 ** 26 + 1) == R.E_ARG
    for name in ("src", "dst", "k", "v", "s", "k2", "v2", "s2"):
        assert copy(R, c, **{name: None}) == R.E_ARG, name
    for name in ("k", "v", "k2", "v2"):
        assert copy(R, c, **{name: P + 8}) == R.E_ARG, name
    for name in ("count", "src", "dst", "rows", "s", "s2"):
        assert copy(R, c, **{name: P + 2}) == R.E_ARG, name
    assert copy(R, c, n=0, src=None, dst=None) == R.OK
    assert copy(R, cfg(R, n_pages=0), k=None) == R.OK and copy(R, c, n_dst=0, k2=None) == R.OK


def test_write_refusals(R):
    c = cfg(R)
    t = lambda **kw: R.write_config(**{**dict(dtype=R.FP16, n_tokens=5, max_new=2, k=(128, 64), v=(128, 64)), **kw})  # noqa: E731
    for kw in (dict(dtype=2), dict(dtype=-1), dict(n_tokens=-1), dict(max_new=-1), dict(k=(-8, 64)), dict(k=(128, 4)),
               dict(v=(12, 64)), dict(v=(128, 2 ** 31))):
        assert write(R, c, t(**kw)) == R.E_ARG, kw
    for name in ("k", "v", "offsets", "held", "table", "k_pages", "v_pages", "scales"):
        assert write(R, c, **{name: None}) == R.E_ARG, name
    for name in ("k", "v", "k_pages", "v_pages"):
        assert write(R, c, **{name: P + 8}) == R.E_ARG, name
    for name in ("offsets", "held", "length", "table", "scales"):
        assert write(R, c, **{name: P + 2}) == R.E_ARG, name
    assert write(R, c, t(n_tokens=0), k=None, v=None) == R.OK
    assert write(R, cfg(R, n_pages=0), k_pages=None, v_pages=None, scales=None) == R.OK
    assert write(R, cfg(R, n_seqs=0), offsets=None, held=None, table=None) == R.OK


def test_attention_refusals(R):
    nan, inf = float("nan"), float("inf")
    c = cfg(R)
    for kw in (dict(dtype=2), dict(heads=0), dict(heads=3), dict(heads=4098), dict(n_q=-1), dict(n_q=2 ** 30), dict(max_q=-1),
               dict(max_k=-1), dict(q=(-8, 64)), dict(q=(256, 4)), dict(out=(256, 12)), dict(scale=nan), dict(scale=inf),
               dict(cap=-1.0), dict(cap=nan), dict(cap=2e38), dict(scale=1e-30, cap=1e30), dict(window=-1), dict(sinks=-1),
               dict(window=5, causal=False)):
        assert attend(R, c, rows_cfg(R, **kw)) == R.E_ARG, kw
    for name in ("q", "offsets", "length", "table", "k", "v", "s", "out"):
        assert attend(R, c, rows_cfg(R), **{name: None}) == R.E_ARG, name
    for name in ("q", "k", "v", "out", "ws"):
        assert attend(R, c, rows_cfg(R), **{name: P + 8}) == R.E_ARG, name
    for name in ("offsets", "start", "length", "prefix", "table", "s", "lse"):
        assert attend(R, c, rows_cfg(R), **{name: P + 2}) == R.E_ARG, name
    assert attend(R, c, rows_cfg(R, n_q=0), q=None, out=None) == R.OK
    assert attend(R, cfg(R, n_seqs=0), rows_cfg(R), offsets=None, length=None, table=None) == R.OK
    with pytest.raises(ValueError):
        rows_cfg(R, scale=None)
    assert rows_cfg(R, scale=None, head_dim=64).scale == 0.125


def test_window_refusals(R):
    def call(window=5, sinks=1, causal=True, n_q=5, **kw):
        c = R.attn_config(4, 2, 64, R.FP16, n_q, 9, (256, 64), (128, 64), (128, 64), (256, 64), 2, 2, 9, causal=causal, **kw)
        return R.rtcc_memory_window_attention(c, window, sinks, P, P, P, P, P, P, None, None, None, None, None, P, None,
                                              None, 0)
    assert call(window=0) == R.E_ARG and call(window=-1) == R.E_ARG and call(sinks=-1) == R.E_ARG
    assert call(causal=False) == R.E_ARG
    assert call(cap=-1.0) == R.E_ARG and call(n_slots=1, slot_rows=9) == R.E_ARG
    assert call(n_q=0) == R.OK
