"""Verification of drafted words (vocab_verify) where what is asked of the kernels is out of the ordinary: many sequences whose next word
comes from the target alone, and logits that are very low or far from zero."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_vocab_verify import Case, _rows  # noqa: E402


def test_a_word_behind_every_draft():
    """All words accepted, or none given: each sequence's next word is drawn from p by its first block, which has one wave look for the
    chunk while the others have yet to see where they are.  The draft of the last sequence ends with its tensor."""
    for dtype, V in (("f32", 500), ("bf16", 9000)):
        c = Case(600, 2, V, dtype, seed=31, short=0.0)
        c.u_accept[:] = 0
        c.drafted[::3] = -1
        n, words = c.check()
        assert (n == np.where(np.arange(600) % 3 == 0, 0, 2)).all()
        for _ in range(20):
            again, more = c.handle.verify(*c.args)
            assert (again.cpu().numpy() == n).all() and (more.cpu().numpy() == words).all()


LOWEST = {"f32": float(np.finfo(np.float32).min), "bf16": -255.0 * 2.0 ** 120}      # (the types' lowest values)


def _with_low_logits(B, T, V, dtype, tau, seed):
    """A batch whose sequences have logits of -1e20, -1e30 or the type's lowest value (a mask's) over whole chunks of a row, over its last
    word, over all words but one, over all of them; and rows far from zero altogether.  (Chunks are of 2048 or 8192 words.)"""
    c = Case(B, T, V, dtype, tau=tau, seed=seed, short=0.1)
    t, d = c.t64.copy(), c.d64.copy()
    whole = V // 8192 * 8192 or V // 2048 * 2048
    for b in range(B):
        low = (-1e20, -1e30, LOWEST[dtype])[b % 3]
        for x, kind in ((t[b], b // 3 % 8), (d[b], b // 24 % 8)):
            if kind == 1:
                x[:, :whole] = low
            elif kind == 2:
                x[:, V - 1] = low
            elif kind == 3:
                x[:, :V // 3] = low
                x[:, V - 1] = low
            elif kind == 4:
                x[:, np.arange(V) != (b * 37) % V] = low
            elif kind == 5:
                x[:] = low
            elif kind == 6:                 # half the words, far below zero; the others further
                x[:] = low / 2
                x[:, ::2] = low / 4
            elif kind == 7:                 # and far above
                x[:, 1::2] = -low / 2
    unit = 4 if dtype == "f32" else 8
    ld = -(-V // unit) * unit
    c.target, c.t64 = _rows(t, dtype, ld)
    c.draft, c.d64 = _rows(d, dtype, ld)
    return c


@pytest.mark.parametrize("tau", [0.5, 0.6, 0.7, 0.8, 0.9, 1.0, 1.2, 1.3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_very_low_logits(dtype, tau):
    """2^((l - m) c) is 1 at the largest logit m of a chunk, whatever m is: c m is not exact, and its rounding past the exponents' range where
    m is the lowest value there is."""
    n, words = _with_low_logits(72, 2, 4097, dtype, tau, seed=41).check()
    assert (words[np.arange(72), n] >= 0).all()


@pytest.mark.parametrize("dtype, tau", [("f32", 0.7), ("f32", 1.0), ("bf16", 0.8), ("bf16", 1.0), ("bf16", 1.3)])
def test_very_low_logits_of_many_rows(dtype, tau):
    """Rows enough for chunks of 8192, of bf16 by the table of powers and what goes past it."""
    B = 600
    n, words = _with_low_logits(B, 1, 8193, dtype, tau, seed=42).check()
    assert (words[np.arange(B), n] >= 0).all()
