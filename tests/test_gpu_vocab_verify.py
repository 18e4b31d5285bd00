"""Verification of drafted words (vocab_verify in include/vocab_ops.h) on the GPU against its float64 oracle.  The results are whole
numbers: they are equal unless a random number lies within rounding of a border, so close (1e-9) that the cases are made without."""
import numpy as np
import pytest

from oracle import serving_oracle as oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1909_00562_amd as lib  # noqa: E402
from paper_1909_00562_amd import binding as bd  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NEAR = 1e-9


def _rows(x, dtype, ld):
    """The logits in rows ld elements apart, NaN between them; (on the GPU, float64)."""
    t = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    wide = torch.full(x.shape[:2] + (ld,), float("nan"), dtype=TYPES[dtype])
    wide[:, :, :x.shape[2]] = t
    return wide.cuda()[:, :, :x.shape[2]], t.double().numpy()


class Case:
    def __init__(self, B, T, V, dtype, tau=1.0, seed=0, wide=0, short=0.3, spread=2.0, off=0.5):
        r = np.random.default_rng(seed + V)
        self.B, self.T, self.V, self.dtype, self.tau = B, T, V, dtype, tau
        base = r.normal(size=(B, T + 1, V)) * spread
        draft = base[:, :T] + r.normal(size=(B, T, V)) * off
        unit = 4 if dtype == "f32" else 8
        ld = -(-V // unit) * unit + wide * unit
        self.target, self.t64 = _rows(base, dtype, ld)
        self.draft, self.d64 = _rows(draft, dtype, ld + unit)
        gumbel = -np.log(-np.log(r.uniform(1e-9, 1, (B, T, V))))
        self.drafted = (self.d64 / tau + gumbel).argmax(axis=2).astype(np.int64)
        for b in range(B):
            if r.uniform() < short:
                self.drafted[b, r.integers(0, T + 1):] = r.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
        self.u_accept, self.u_next = r.uniform(size=(B, T)).astype(np.float32), r.uniform(size=B).astype(np.float32)

    def run(self, h=None):
        h = h or lib.DeviceVocabVerify(self.B, self.T, self.V, dtype=self.dtype, temperature=self.tau)
        up = lambda x, t: torch.from_numpy(x.astype(t)).cuda()  # noqa: E731
        self.args = (self.target, self.draft, up(self.drafted, np.int32), up(self.u_accept, np.float32), up(self.u_next, np.float32))
        self.handle = h
        n, w = h.verify(*self.args)
        return n.cpu().numpy(), w.cpu().numpy()

    def want(self):
        got = [oracle.verify(self.t64[b], self.d64[b], self.drafted[b], self.u_accept[b], self.u_next[b], self.tau) for b in range(self.B)]
        return np.array([g[0] for g in got]), np.array([g[1] for g in got])

    def off_borders(self):
        """Moves random numbers that lie within rounding of a border."""
        for b in range(self.B):
            while True:
                n, words = oracle.verify(self.t64[b], self.d64[b], self.drafted[b], self.u_accept[b], self.u_next[b], self.tau)
                near = False
                for t in range(min(n + 1, self.T)):
                    x = self.drafted[b, t]
                    if 0 <= x < self.V:
                        p, q = oracle.softmax(self.t64[b, t], self.tau), oracle.softmax(self.d64[b, t], self.tau)
                        if p is not None and q is not None and abs(float(self.u_accept[b, t]) * q[x] - p[x]) < NEAR * p[x]:
                            self.u_accept[b, t], near = np.float32(self.u_accept[b, t] * 0.99), True
                p = oracle.softmax(self.t64[b, n], self.tau)
                if p is not None and words[n] >= 0:
                    given = n < self.T and 0 <= self.drafted[b, n] < self.V
                    rest = np.maximum(p - (oracle.softmax(self.d64[b, n], self.tau) if given else 0), 0)
                    rest = rest if rest.sum() > 0 else p
                    sums = np.cumsum(rest) / rest.sum()
                    at = float(self.u_next[b])
                    if 0 < at < 1 and np.abs(sums - at).min() < NEAR:
                        self.u_next[b], near = np.float32(at * 0.99), True
                if not near:
                    break
        return self

    def check(self):
        self.off_borders()
        n, words = self.run()
        want_n, want_words = self.want()
        assert (n == want_n).all() and (words == want_words).all(), (n, want_n, words, want_words)
        return n, words


@pytest.mark.parametrize("B, T, V, dtype, tau, wide", [
    (1, 1, 1, "f32", 1.0, 0), (1, 1, 2, "bf16", 1.0, 1), (7, 3, 5, "f32", 0.5, 0), (33, 4, 100, "bf16", 1.0, 0), (9, 5, 8191, "f32", 0.7, 2),
    (9, 2, 8192, "bf16", 1.3, 0), (9, 5, 8193, "bf16", 1.0, 0), (5, 64, 1003, "f32", 1.0, 0), (16, 4, 32003, "bf16", 0.9, 0), (3, 8, 128000, "f32", 1.0, 0),
    (2, 1, 1 << 20, "bf16", 1.0, 0), (300, 1, 17, "bf16", 2.0, 0), (30000, 1, 3, "f32", 1.0, 0)])
def test_words(B, T, V, dtype, tau, wide):
    Case(B, T, V, dtype, tau, seed=B, wide=wide).check()


def test_all_of_a_draft_or_none_of_it():
    c = Case(40, 3, 500, "f32", seed=3, short=0.0)
    c.u_accept[:] = 0
    n, _ = c.check()
    assert (n == 3).all()
    c = Case(40, 3, 500, "f32", seed=4, short=0.0, off=0.0)        # a draft from the target itself
    c.u_accept[:] = np.float32(1 - 2.0 ** -24)
    n, _ = c.check()
    assert (n == 3).all()
    c = Case(40, 3, 500, "f32", seed=5, short=1.0)
    c.drafted[:] = -1
    n, _ = c.check()
    assert (n == 0).all()
    c = Case(40, 3, 500, "bf16", seed=6, short=0.0, spread=0.1, off=9.0)
    c.u_accept[:] = np.float32(0.999)
    n, _ = c.check()
    assert (n == 0).any()


def test_random_numbers_at_the_ends():
    for u in (0.0, 1 - 2.0 ** -24, 1.0, -0.5):
        c = Case(12, 2, 9000, "f32", seed=8)
        c.u_next[:] = u
        _, words = c.check()
        assert (words[np.arange(12), c.want()[0]] >= 0).all()


def test_words_of_no_probability():
    """-inf in either row: an excluded word is refused, and is never drawn; one that only the target has is drawn."""
    B, V = 64, 40
    c = Case(B, 2, V, "f32", seed=9, short=0.0)
    r = np.random.default_rng(0)
    t, d = c.t64.copy(), c.d64.copy()
    t[:, :, r.permutation(V)[:30]] = -np.inf
    d[::2, :, 5:] = -np.inf
    c.target, c.t64 = _rows(t, "f32", V)
    c.draft, c.d64 = _rows(d, "f32", V)
    c.drafted[::2] %= 5
    n, words = c.check()
    for b in range(B):
        assert np.isfinite(c.t64[b, n[b], words[b, n[b]]])
    # one word alone is left
    t = np.full_like(t, -np.inf)
    t[:, :, 33] = -4.0
    c.target, c.t64 = _rows(t, "f32", V)
    n, words = c.check()
    assert (words[np.arange(B), n] == 33).all()


def test_rows_that_are_no_distributions():
    for bad in (np.nan, np.inf, -np.inf):
        c = Case(16, 3, 20000, "f32", seed=11, short=0.0)
        c.u_accept[:] = 0                                   # (all accepted, were it not for these)
        t, d = c.t64.copy(), c.d64.copy()
        for b in range(16):
            x = d[b, b % 3] if b % 2 else t[b, b % 4]
            x[slice(None) if bad == -np.inf else 17000] = bad
        c.target, c.t64 = _rows(t, "f32", 20000)
        c.draft, c.d64 = _rows(d, "f32", 20000)
        n, words = c.run()
        want_n, want_words = c.want()
        assert (n == want_n).all() and (words == want_words).all()
        assert (words[np.arange(16), n] == -1).all()
    # rows that nobody asks for may hold anything
    c = Case(8, 3, 300, "bf16", seed=12, short=0.0)
    c.drafted[:, 1] = -1
    t, d = c.t64.copy(), c.d64.copy()
    t[:, 2:], d[:, 1:] = np.nan, np.nan
    c.target, c.t64 = _rows(t, "bf16", 304)
    c.draft, c.d64 = _rows(d, "bf16", 304)
    n, words = c.check()
    assert (words[np.arange(8), n] >= 0).all()


def test_words_are_drawn_as_the_target_says():
    """Many draws of one pair of rows: the first word of each is distributed as p.  (Chi-square: V - 1 degrees, 6 standard deviations.)"""
    B, V = 40000, 6
    r = np.random.default_rng(2)
    p, q = np.array([0.3, 0.05, 0.25, 0.1, 0.2, 0.1]), np.array([0.1, 0.3, 0.1, 0.2, 0.1, 0.2])
    t = torch.from_numpy(np.log(p)).float().cuda().expand(B, 2, V)
    rows = torch.zeros(B, 2, 8, device="cuda")
    rows[:, :, :V] = t
    d = torch.zeros(B, 1, 8, device="cuda")
    d[:, :, :V] = torch.from_numpy(np.log(q)).float().cuda()
    drafted = torch.from_numpy(r.choice(V, size=(B, 1), p=q).astype(np.int32)).cuda()
    u, v = (torch.from_numpy(r.uniform(size=s).astype(np.float32)).cuda() for s in ((B, 1), (B,)))
    n, words = lib.DeviceVocabVerify(B, 1, V, dtype="f32").verify(rows[:, :, :V], d[:, :, :V], drafted, u, v)
    count = np.bincount(words[:, 0].cpu().numpy(), minlength=V)
    chi = ((count - B * p) ** 2 / (B * p)).sum()
    assert chi < (V - 1) + 6 * np.sqrt(2 * (V - 1))
    assert abs(float((n == 1).float().mean()) - np.minimum(p, q).sum()) < 6 * 0.5 / np.sqrt(B)


def test_calls_are_alike_and_captured():
    c = Case(21, 4, 20003, "bf16", seed=13).off_borders()
    n, words = c.run()
    h, out = c.handle, [torch.empty(21, dtype=torch.int32, device="cuda"), torch.empty(21, 5, dtype=torch.int32, device="cuda")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h.verify(*c.args, *out)
    for i in range(5):
        for t in out:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert (out[0].cpu().numpy() == n).all() and (out[1].cpu().numpy() == words).all()
        again, more = h.verify(*c.args)
        assert (again.cpu().numpy() == n).all() and (more.cpu().numpy() == words).all()


def test_refusals_of_the_handle():
    h = lib.DeviceVocabVerify(2, 3, 16, dtype="f32")
    t, d = torch.zeros(2, 4, 16, device="cuda"), torch.zeros(2, 3, 16, device="cuda")
    x, u, v = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, device="cuda"), torch.zeros(2, device="cuda")
    h.verify(t, d, x, u, v)
    wide = torch.zeros(2, 4, 18, device="cuda")
    for args, code in (((t.bfloat16(), d, x, u, v), 3), ((t[:, :3], d, x, u, v), 2), ((t, d, x.long(), u, v), 3), ((t, d, x, u.cpu(), v), 2),
                       ((wide[:, :, :16], d, x, u, v), 5), ((t.transpose(0, 1).contiguous().transpose(0, 1), d, x, u, v), 5), ((t, None, x, u, v), 1)):
        with pytest.raises(bd.AttnSoftmaxError) as e:
            h.verify(*args)
        assert e.value.code == code


@pytest.mark.parametrize("tau", [1.0, 0.1, 0.09])
def test_many_rows_of_bf16(tau):
    """Enough chunks for the table of powers (0.09: a temperature past its range), and logits that are not in it: zeros, tiny and large ones, -inf;
    rows that are no distributions; short drafts whose further rows hold NaN."""
    c = Case(70, 4, 40003, "bf16", tau=tau, seed=20, spread=2.0 * tau, off=0.4 * tau)
    t, d = c.t64.copy(), c.d64.copy()
    t[3, 1, 5:9], t[4, 0, 40000], t[5, 2, ::2], t[6, 3, 77] = 0.0, 1e-7, -np.inf, 300.0 * tau
    d[3, 0, 39999], d[4, 1, 100:9000], d[5, 0, 1::2], d[6, 2, 9] = -1e-30, 0.0, -np.inf, 70.0 * tau
    t[7, 0, 3], t[8, 1, 12000], d[9, 0, 40002] = np.nan, np.inf, np.nan
    t[10] = 0.0
    d[10] = 0.0
    c.drafted[11, 2:] = -1
    t[11, 3:], d[11, 2:] = np.nan, np.nan
    unit = -(-c.V // 8) * 8
    c.target, c.t64 = _rows(t, "bf16", unit)
    c.draft, c.d64 = _rows(d, "bf16", unit + 8)
    n, words = c.check()
    assert words[7, 0] == -1 and n[7] == 0 and n[9] == 0
