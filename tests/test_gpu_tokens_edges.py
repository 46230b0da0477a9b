"""Token memory at its edges: sizes near 2^31, scores and caps far from the usual
ones, non-finite values, slots that fill up, hints that are too small, and what
happens when a launch or a wait fails.

Tolerances are those of test_gpu_tokens.py (u: the storage type's unit roundoff,
d: a score's error, A = sum_j p_j |v_j|), unless a test derives its own.
"""
import numpy as np
import pytest

from tests import gpu_util as U

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
