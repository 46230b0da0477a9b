"""Token-memory entry points without a GPU: every refusal comes before any GPU
work, empty calls succeed, and the configuration helpers fill the structs."""
import ctypes

import pytest

from paper_2608_08330_gb300 import build as B


@pytest.fixture(scope="module")
def R():
    B.build()
    from paper_2608_08330_gb300 import rtcc
    rtcc.load()
    return rtcc


P = 0x10000            # an aligned address; refused calls never read it


def append(R, n_seqs=3, capacity=10, n_tokens=5, **kw):
    a = dict(new=P, held=P + 64, slot=None, offsets=P + 128, rows=P, seq=None, pos=None, begin=P, end=P,
             length=P + 256)
    a.update(kw)
    return R.rtcc_memory_append(n_seqs, capacity, n_tokens, *a.values())


def test_append_refusals(R):
    assert append(R, n_seqs=-1) == R.E_ARG
    assert append(R, n_seqs=16385) == R.E_ARG
    assert append(R, capacity=0) == R.E_ARG
    assert append(R, n_tokens=-1) == R.E_ARG
    for name in ("new", "held", "offsets", "rows", "begin", "end", "length"):
        assert append(R, **{name: None}) == R.E_ARG, name
        assert append(R, **{name: P + 2}) == R.E_ARG, name
    for name in ("slot", "seq", "pos"):
        assert append(R, **{name: P + 1}) == R.E_ARG, name
    assert append(R, length=P + 64) == R.E_ARG          # over d_held
    assert append(R, length=P) == R.E_ARG               # over d_new


def prep_cfg(R, **kw):
    a = dict(heads=4, kv_heads=2, head_dim=64, dtype=R.FP16, n_tokens=7, n_rows=9, q=(256, 64), k=(128, 64), v=(128, 64),
             q_out=(256, 64), k_mem=(128, 64), v_mem=(128, 64), axis_pairs=(8, 12, 12))
    a.update(kw)
    return R.prepare_config(**a)


def prepare(R, cfg, **kw):
    a = dict(q=P, k=P, v=P, q_gain=None, k_gain=None, pos=P, rows=None, q_out=P, k_mem=P, v_mem=P, coord=None)
    a.update(kw)
    return R.rtcc_qkv_prepare(cfg, *a.values())


def test_prepare_refusals(R):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(dtype=2), dict(n_tokens=-1), dict(n_rows=-1), dict(heads=-1), dict(kv_heads=-2), dict(heads=0),
               dict(kv_heads=0), dict(heads=4097), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136),
               dict(axis_pairs=(-1, 3, 3)), dict(axis_pairs=(20, 12, 1)), dict(axis_pairs=(2 ** 31 - 1, 0, 0)),
               dict(theta=0.5), dict(theta=nan), dict(theta=inf), dict(eps=-1e-3), dict(eps=nan),
               dict(q=(250, 64)), dict(k=(128, 60)), dict(v=(-8, 64)), dict(q_out=(256, 4)), dict(k_mem=(12, 64)),
               dict(v_mem=(128, -64))):
        assert prepare(R, prep_cfg(R, **kw)) == R.E_ARG, kw
    cfg = prep_cfg(R)
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_mem=None), dict(v=None), dict(v_mem=None),
               dict(pos=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(q_out=P + 8), dict(k_mem=P + 8),
               dict(v_mem=P + 8), dict(coord=P + 4), dict(pos=P + 2), dict(rows=P + 1), dict(q_gain=P + 2),
               dict(k_gain=P + 2)):
        assert prepare(R, cfg, **kw) == R.E_ARG, kw
    assert R.load().rtcc_qkv_prepare(None, *[None] * 12) == R.E_ARG


def test_prepare_of_nothing_is_ok(R):
    assert prepare(R, prep_cfg(R, n_tokens=0)) == R.OK
    assert prepare(R, prep_cfg(R), q=None, q_out=None, k=None, k_mem=None, v=None, v_mem=None) == R.OK


def attn_cfg(R, **kw):
    a = dict(heads=4, kv_heads=2, head_dim=64, dtype=R.BF16, n_q=7, n_rows=90, q=(256, 64), k=(128, 64), v=(128, 64),
             out=(256, 64), n_seqs=2, max_q=4, max_k=50)
    a.update(kw)
    return R.attn_config(**a)


def attend(R, cfg, **kw):
    a = dict(q=P, k=P, v=P, q_offsets=P, k_begin=P, k_end=P, prefix=None, present=None, slopes=None, q_pos=None,
             k_pos=None, out=P, lse=None, workspace=None, workspace_bytes=0)
    a.update(kw)
    return R.rtcc_memory_attention(cfg, *a.values())


def test_attention_refusals(R):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(dtype=-1), dict(heads=0), dict(heads=5), dict(kv_heads=0), dict(heads=8192, kv_heads=1),
               dict(head_dim=4), dict(head_dim=65), dict(head_dim=256), dict(n_q=-1), dict(n_rows=-1), dict(n_seqs=-1),
               dict(max_q=-1), dict(max_k=-1), dict(n_q=2 ** 30), dict(q=(252, 64)), dict(k=(128, 1)), dict(v=(4, 64)),
               dict(out=(256, -8)), dict(scale=nan), dict(scale=inf), dict(cap=-1.0), dict(cap=nan),
               dict(n_slots=2, slot_rows=45), dict(n_slots=-1)):
        assert attend(R, attn_cfg(R, **kw)) == R.E_ARG, kw
    for kw in (dict(n_slots=65, slot_rows=90), dict(n_slots=2, slot_rows=0), dict(n_slots=2, slot_rows=44), dict()):
        assert attend(R, attn_cfg(R, **kw), present=P) == R.E_ARG, kw
    cfg = attn_cfg(R)
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_offsets=None), dict(k_begin=None),
               dict(k_end=None), dict(slopes=P), dict(q_pos=P, k_pos=P), dict(slopes=P, q_pos=P), dict(q=P + 8),
               dict(k=P + 8), dict(v=P + 2), dict(out=P + 4), dict(workspace=P + 8), dict(lse=P + 2),
               dict(q_offsets=P + 2), dict(prefix=P + 3), dict(slopes=P, q_pos=P, k_pos=P + 4)):
        assert attend(R, cfg, **kw) == R.E_ARG, kw
    assert attend(R, attn_cfg(R, q_pos_row=1), slopes=P, q_pos=P, k_pos=P) == R.E_ARG
    assert R.load().rtcc_memory_attention(None, *[None] * 14, 0, None) == R.E_ARG


def test_attention_of_nothing_is_ok(R):
    assert attend(R, attn_cfg(R, n_q=0), q=None, out=None) == R.OK
    assert attend(R, attn_cfg(R, n_seqs=0), q_offsets=None, k_begin=None, k_end=None) == R.OK


def test_config_helpers_match_the_struct(R):
    c = prep_cfg(R, interleaved=True, norm=False, theta=100.0, eps=1e-5)
    assert (c.heads, c.kv_heads, c.head_dim, c.qo_row, c.vm_head) == (4, 2, 64, 256, 64)
    assert list(c.axis_pairs) == [8, 12, 12] and c.interleaved == 1 and c.norm == 0
    a = attn_cfg(R, causal=True, cap=30.0)
    assert a.scale == ctypes.c_float(0.125).value and a.cap == 30.0 and a.causal == 1 and a.q_pos_row == 2


def test_check_raises_with_the_status(R):
    assert R.check(R.OK) == R.OK
    with pytest.raises(R.RTCCError) as e:
        R.check(R.E_ARG, "rtcc_memory_attention")
    assert e.value.status == R.E_ARG
