"""Attention over the paged cache where scores are far from zero: the greatest ones take all, and equal ones share, whatever their size."""
import numpy as np
import pytest

from oracle import serving_oracle as oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1909_00562_amd as lib  # noqa: E402
from test_gpu_kv_cache import BF, CACHES, TYPES, U, Attn  # noqa: E402


def _levels(lengths, T, heads, G, D, dtype, cache, size, window=0, max_len=None, seed=0):
    """Keys that are signs, the same of each head, times 1, -1 or half of that; queries these signs times a number of 8 bits, every other one the other
    way round: the greatest scores are about `size`, those of a sequence in two about -size / 2, and all but equal ones are size / 2 apart.
    Sums of them are exact in fp32 (127 or 7 times 255 times D <= 256, and a power of two), so that equal keys have equal scores."""
    c = Attn(lengths, T, heads, G, D, 16, dtype, cache, window, seed=seed, max_len=max_len)
    r = np.random.default_rng(seed)
    signs = np.where(r.uniform(size=(heads, D)) < 0.5, -1.0, 1.0)
    for b, n in enumerate(lengths):
        level = r.choice([1.0, -1.0, 0.5, -0.5] if b % 2 == 0 else [-1.0, -0.5], size=n)
        for i in range(n):
            got = c.pool.put(b, i, (signs * level[i]).astype(np.float32), _values_of(r, heads, D, dtype))
            if got is not None:
                c.k[b][i], c.v[b][i] = got
    c.c = c.pool.device()
    c.h = lib.DeviceKvAttn(c.c, len(lengths), T, heads * G, c.max_len, window=window)
    power = 2.0 ** np.round(np.log2(size / (D * c.scale)))
    q = np.repeat(signs, G, axis=0) * np.where(np.arange(heads * G) % 2, -power, power)[:, None]
    q = q * (2 * r.integers(64, 128, (len(lengths), T, heads * G, 1)) + 1) / 128
    q = torch.from_numpy(q.astype(np.float32)).to(TYPES[dtype])
    c.q, c.q64 = q.cuda(), q.double().numpy()
    return c


def _values_of(r, heads, D, dtype):
    return torch.from_numpy(r.normal(size=(heads, D)).astype(np.float32)).to(TYPES[dtype]).float().numpy()


def _check(c):
    """Weights are 1 or 0 before they are divided by their sum, and held as two bf16 terms (2^-16) or three or one (2^-22); sums of n weights and
    values are off by 4 (n + 8) u of their magnitudes; the log-sum-exp by the roundings of score, scale and product, at most 8 u of it."""
    for b, n in enumerate(c.lengths):
        o, lse = oracle.attn(c.q64[b], c.k[b], c.v[b], c.there[b], c.scale, c.window)
        mag, _ = oracle.attn(c.q64[b], c.k[b], np.abs(c.v[b]), c.there[b], c.scale, c.window)
        rel = 4 * (n + 8) * U + (2.0 ** -16 if c.dtype == "bf16" else 2.0 ** -22)
        bound = rel * mag + (BF if c.dtype == "bf16" else 0) * (np.abs(o) + rel * mag)
        out, got = c.out[b].double().cpu().numpy(), c.lse[b].double().cpu().numpy()
        assert (np.abs(out - o) <= bound).all(), (b, np.abs(out - o).max())
        some = ~np.isneginf(lse)
        assert (np.isneginf(got) == ~some).all()
        assert (np.abs(got[some] - lse[some]) <= 8 * U * np.abs(lse[some]) + 4 * (n + 8) * U).all()


@pytest.mark.parametrize("size", [1e8, 1e10, 1e20])
@pytest.mark.parametrize("dtype, cache", CACHES)
@pytest.mark.parametrize("lengths, T, heads, G, D, window, max_len", [
    ([1, 1], 1, 1, 2, 16, 0, None), ([70, 33, 5, 16], 1, 2, 2, 64, 0, None), ([120, 50], 5, 1, 8, 128, 40, None), ([40, 70], 2, 1, 2, 256, 0, None),
    ([700, 300, 3], 1, 1, 2, 64, 0, 9000), ([i * 5 % 13 for i in range(120)], 2, 11, 2, 32, 0, 9000)])
def test_large_scores(dtype, cache, lengths, T, heads, G, D, window, max_len, size):
    """The weight of the greatest score is 1: a scaled score minus the rounded maximum of scaled scores is no 0 there, and past 2^31 it leaves the
    exponential's range.  One block, several that are joined, and more of them than runs."""
    c = _levels(lengths, T, heads, G, D, dtype, cache, size, window, max_len, seed=D)
    _check(c.run())
