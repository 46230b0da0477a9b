"""Refusals of the token-memory calls at the edges of their ranges, without a GPU."""
import pytest

from tests.test_tokens_cpu import P, attend, attn_cfg, prep_cfg, prepare
from paper_2608_08330_gb300 import build as B


@pytest.fixture(scope="module")
def R():
    B.build()
    from paper_2608_08330_gb300 import rtcc
    rtcc.load()
    return rtcc


def test_attention_refuses_row_numbers_that_would_wrap(R):
    limit = 2 ** 31 - 2 ** 16
    for kw in (dict(n_rows=limit + 1), dict(n_rows=2 ** 31 - 1), dict(n_q=limit // 4 + 1), dict(n_q=(2 ** 31 - 1) // 4)):
        assert attend(R, attn_cfg(R, **kw)) == R.E_ARG, kw
    # a call of the largest sizes with nothing to do is none of these
    assert attend(R, attn_cfg(R, n_rows=limit, n_q=limit // 4, n_seqs=0)) == R.OK
    assert attend(R, attn_cfg(R, n_rows=limit, n_q=0), q=None, out=None, present=P) == R.E_ARG    # no slots given


def test_attention_refuses_caps_out_of_range(R):
    for kw in (dict(cap=1.1e38), dict(cap=1e30, scale=1e-19), dict(cap=1e-38, scale=100.0)):
        assert attend(R, attn_cfg(R, **kw)) == R.E_ARG, kw
    for kw in (dict(cap=1e38, scale=2.0), dict(cap=1e30, scale=0.0), dict(cap=1e-38, scale=1.0)):
        assert attend(R, attn_cfg(R, n_seqs=0, **kw)) == R.OK, kw


def test_attention_start_is_checked_and_passed_on(R):
    c = attn_cfg(R, causal=True, q_start=P + 64)
    assert c.d_q_start == P + 64 and attn_cfg(R).d_q_start is None
    assert attend(R, attn_cfg(R, causal=True, q_start=P + 2)) == R.E_ARG


def test_attention_test_hook_refuses_unknown_bits(R):
    assert R.rtcc_test_attention(1 << 20) == R.E_ARG and R.rtcc_test_attention(-1) == R.E_ARG
    assert R.rtcc_test_attention(R.TEST_UNREACHABLE_WAIT) == R.OK and R.rtcc_test_attention(0) == R.OK


def test_prepare_needs_positions_to_turn_or_keep_them(R):
    plain = prep_cfg(R, axis_pairs=(0, 0, 0))
    assert prepare(R, plain, pos=None, coord=P) == R.E_ARG
    assert prepare(R, prep_cfg(R), pos=None) == R.E_ARG
    assert prepare(R, prep_cfg(R, axis_pairs=(0, 0, 0), n_tokens=0), pos=None) == R.OK
