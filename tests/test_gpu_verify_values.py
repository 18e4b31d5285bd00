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
