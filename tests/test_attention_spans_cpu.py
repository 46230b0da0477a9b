"""The numbering of keys that the attention kernels share (attn.cuh), compiled for the
host: which tokens a sequence has, which keys each of them sees and in which rows, against
the definition, and that no number lies past the room that the host makes for it.
"""
import ctypes as C
import os
import random
import subprocess

import numpy as np
import pytest

from paper_2608_08330_gb300 import build as B

SOURCE = r"""
#include "attn.cuh"

// out: first token, tokens, keys, room; rows: the row of every key; per token what it sees
// of keys from afar, where its window begins, and the end of its keys.
extern "C" void span(int causal, int window, int sinks, int n_q, int n_rows, int most_q, int most_k,
                     const int* q_offsets, const int* k_begin, const int* k_end, const int* prefix,
                     const int* q_start, int seq, int* out, int* rows, int n_out, int* sees) {
  rtcc::AttnArgs a{};
  a.causal = causal; a.window = window; a.sinks = sinks; a.n_q = n_q; a.n_rows = n_rows;
  a.most_q = most_q; a.most_k = most_k;
  a.q_offsets = q_offsets; a.k_begin = k_begin; a.k_end = k_end; a.prefix = prefix; a.q_start = q_start;
  const rtcc::AttnSpan s = rtcc::attn_span<true>(a, seq);
  out[0] = s.q0; out[1] = s.nq; out[2] = s.nk;
  out[3] = (int)rtcc::attn_most_keys(a, most_q < 1 ? 1 : most_q, most_k < 1 ? 1 : most_k);
  for (int j = 0; j < s.nk && j < n_out; ++j) rows[j] = rtcc::attn_row(s, j);
  for (int i = 0; i < s.nq; ++i) {
    const rtcc::AttnView v = rtcc::attn_view(a, s, s.first, i);
    sees[3 * i] = v.seen;
    sees[3 * i + 1] = v.low;
    sees[3 * i + 2] = rtcc::attn_visible(a, s, s.first, i);
  }
}
"""


@pytest.fixture(scope="module")
def span(tmp_path_factory):
    d = tmp_path_factory.mktemp("span")
    (d / "span.cu").write_text(SOURCE)
    cuda = B._cuda_home()
    subprocess.run([os.path.join(cuda, "bin", "nvcc")] + B.ARCH + ["-O1", "-std=c++17", "--expt-relaxed-constexpr", "-shared",
                   "-Xcompiler", "-fPIC", "-I" + B.CSRC, "-I" + B.INCLUDE, str(d / "span.cu"), "-o", str(d / "span.so")],
                   check=True)
    lib = C.CDLL(str(d / "span.so"))

    def call(offsets, begin, end, seq, causal=1, window=0, sinks=0, prefix=None, start=None, n_q=None, n_rows=0, most_q=0,
             most_k=0):
        """(first token, tokens, keys, room, row of each key, [token][seen, low, end])"""
        arr = lambda v: None if v is None else (C.c_int * len(v))(*v)  # noqa: E731
        out, rows, sees = (C.c_int * 4)(), (C.c_int * 4096)(), (C.c_int * (3 * 4096))()
        lib.span(causal, window, sinks, offsets[-1] if n_q is None else n_q, n_rows, most_q, most_k, arr(offsets), arr(begin),
                 arr(end), arr(prefix), arr(start), seq, out, rows, 4096, sees)
        q0, nq, nk, room = out
        return q0, nq, nk, room, np.array(rows[:nk]), np.array(sees[:3 * nq]).reshape(nq, 3)

    return call


def rows_seen(nk, rows, see, window):
    """The rows that one token sees, from its three numbers."""
    j = np.arange(nk)
    on = j < see[2]
    if window:
        on = on & ((j < see[0]) | (j >= see[1]))
    return rows[on]


def definition(m, p, causal, window, sinks, prefix):
    """Keys that the token at place p sees of m."""
    j = np.arange(m)
    if not causal:
        return j
    see = j <= p
    if window:
        see = see & ((j > p - window) | (j < sinks))
    return j[see | (j < prefix)]


def sizes(rng, most):
    return rng.choice([0, 1, 63, 64, 65, rng.randint(0, most), rng.randint(0, most)])


def test_pages_tokens_past_the_limit_take_their_keys_along(span):
    """A sequence of more tokens than max_q: those kept see what the definition says, and keys
    that only left-out tokens would see are not among the sequence's, so that they fit the room
    that the host makes for max_q tokens."""
    rng = random.Random(1)
    cut = 0
    for _ in range(3000):
        n, m = sizes(rng, 900), sizes(rng, 2000)
        window = rng.choice([0, 1, 64, rng.randint(1, 300), rng.randint(1, 3000)])
        sinks = rng.choice([0, 1, 64, rng.randint(0, 200)])
        prefix = rng.choice([None, None, 0, rng.randint(0, m)])
        start = rng.choice([None, rng.randint(0, max(0, m))])
        causal = 1 if window else rng.choice([0, 1, 1])
        most_q = rng.choice([0, 1, n, max(0, n - 1), rng.randint(0, n)])
        q0, nq, nk, room, rows, sees = span([3, 3 + n], None, [m], 0, causal, window, sinks,
                                            None if prefix is None else [prefix], None if start is None else [start],
                                            most_q=most_q, most_k=m)
        assert (q0, nq) == (3, min(n, most_q))
        assert nk <= (room if window else m), (n, m, window, sinks, start, most_q)
        first = start if start is not None and causal else m - n
        for i in range(nq):
            want = definition(m, first + i, causal, window, sinks, prefix or 0)
            assert rows_seen(nk, rows, sees[i], window).tolist() == want.tolist()
        if nq and causal:
            assert nk == sees[:, 2].max()
            cut += nq < n
    assert cut > 500


def test_pages_many_left_out_tokens_stay_within_the_room(span):
    """100,000 tokens of which 2,000 are taken, windows of 100: the keys of 2,000."""
    q0, nq, nk, room, rows, sees = span([0, 100000], None, [100000], 0, 1, 100, 0, most_q=2000, most_k=100000)
    assert nq == 2000 and nk <= room == 100 + 2000 + 63


@pytest.mark.parametrize("pages", [False, True])
def test_places_are_what_they_are_given_as(span, pages):
    """A token is at the place that its start says, behind the span's end too, and, without
    starts, counts from the sequence's own length, not from what max_k leaves of it."""
    rng = random.Random(2 + pages)
    behind = cut = 0
    for _ in range(4000):
        n, m = rng.choice([1, 2, 40, rng.randint(0, 400)]), sizes(rng, 1500)
        window = rng.choice([0, 1, 64, rng.randint(1, 300), rng.randint(1, 3000), 2 ** 31 - 1])
        sinks = rng.choice([0, 1, 64, rng.randint(0, 200), 2 ** 31 - 1])
        prefix = rng.choice([None, None, 0, rng.randint(0, m), m + 7])
        start = rng.choice([None, rng.randint(0, m), m, m + rng.randint(0, 500), 2 ** 31 - 1])
        most_k = rng.choice([m, m + 9, rng.randint(0, m), 64]) if pages else m
        kw = dict(prefix=None if prefix is None else [prefix], start=None if start is None else [start], most_q=n)
        if pages:
            _, nq, nk, room, rows, sees = span([0, n], None, [m], 0, 1, window, sinks, most_k=most_k, **kw)
        else:
            _, nq, nk, room, rows, sees = span([0, n], [5], [5 + m], 0, 1, window, sinks, n_rows=5 + m, most_k=max(m, 1), **kw)
        assert nq == n and nk <= max(0, min(m, room))
        have = min(m, most_k)
        first = m - n if start is None else start
        for i in range(n):
            want = [j for j in definition(m, first + i, True, window, sinks, prefix or 0) if j < have]
            got = rows_seen(nk, rows, sees[i], window) - (0 if pages else 5)
            assert got.tolist() == want, (n, m, window, sinks, prefix, start, most_k, i)
        behind += window > 0 and n > 0 and first > have
        cut += have < m
    assert behind > 300 and (cut > 300 or not pages)
