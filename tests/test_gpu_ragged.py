"""Attention of many sequences of unlike lengths in one call, where spans are split and
partial results merged: every row of the merge finds its own sequence.  Tolerances as in
test_gpu_tokens.py.
"""
import numpy as np
import pytest

from tests import gpu_util as U
from tests.test_gpu_tokens import Case, i32

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def R():
    return U.load()


def lengths(count, longest, rng):
    """One long sequence at a place of its own, empty ones, runs of them, single tokens."""
    n = [int(x) for x in rng.choice([0, 0, 1, 1, 2, 7], count)]
    n[rng.integers(count)] = longest
    return n


# 100 tokens are one tile of 128 rows: its two chains share it, and their results are merged
@pytest.mark.parametrize("count", [1, 2, 31, 32, 33, 64, 65, 1000])
@pytest.mark.parametrize("heads,kv,dim,dtype", [(3, 3, 64, "fp16"), (4, 2, 128, "bf16")])
@pytest.mark.parametrize("causal", [False, True])
def test_ragged_merges(R, count, heads, kv, dim, dtype, causal):
    rng = np.random.default_rng(count)
    n = lengths(count, 100, rng)
    m = [x + int(rng.choice([0, 0, 5, 130])) for x in n]
    Case(n, m, heads, kv, dim, dtype, causal=causal).run(R, workspace=64 << 20).check()


@pytest.mark.parametrize("count", [3, 40])
def test_ragged_merges_of_many_parts(R, count):
    """Few tokens over long spans, in more parts than a cluster joins."""
    rng = np.random.default_rng(count)
    n = [int(x) for x in rng.choice([0, 1, 3], count)]
    n[0], n[-1] = 2, 1
    m = [int(x) for x in rng.choice([0, 20, 700, 9000], count)]
    m[-1] = 90000
    Case(n, m, 2, 1, 64).run(R, workspace=64 << 20).check()
    Case(n, m, 4, 4, 128, "bf16", causal=True).run(R, workspace=64 << 20, max_q=1, max_k=60000).check()


@pytest.mark.parametrize("count", [1, 33, 70])
def test_ragged_tokens_of_no_sequence(R, count):
    """Tokens before the first offset and from the last one on are left as they were."""
    rng = np.random.default_rng(count)
    n = lengths(count, 100, rng)
    n[0], n[-1] = n[0] + 4, n[-1] + 3
    m = [200] * count
    c = Case(n, m, 2, 2, 64).run(R).check()
    whole, lse = c.out.clone(), c.lse.clone()
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    off[0] += 2
    off[-1] -= 1
    c.out.fill_(7)
    c.lse.fill_(7)
    c.run(R, off=i32(off))
    torch.cuda.synchronize()
    for t, w in ((c.out, whole), (c.lse, lse)):
        assert bool((t[:2] == 7).all()) and bool((t[-1:] == 7).all())
        t[:2], t[-1:] = w[:2], w[-1:]
    c.check()
