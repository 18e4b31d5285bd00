"""The paged cache and the attention over it (include/kv_cache.h) on the GPU against their float64 oracle.

Codes and what they stand for are exact.  Attention: u = 2^-24 is half a step of fp32, 2^-8 of bf16.  A score is off by ds = 2 (D + 8) u
sum |q k| scale + 8 u |score| (a sum of D fp32 products, its factors); a weight by e^ds, and by 4 u for the exponential and its argument's
rounding, (2 + |score - max|) u; sums of n weights and of n products by 2 (n + 8) u of their magnitudes; weights as two bf16 terms by 2^-16, as
three by 2^-24."""
import numpy as np
import pytest

from oracle import serving_oracle as oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1909_00562_amd as lib  # noqa: E402
from paper_1909_00562_amd import binding as bd  # noqa: E402

U, BF = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
GUARD = 64


def _guarded(shape, dtype):
    n = int(np.prod(shape))
    base = torch.full((n + GUARD,), 7.0, device="cuda", dtype=dtype)
    return base, base[:n].view(*shape)


def _bits(t):
    return t.contiguous().view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.element_size()])


def _same_bits(a, b):
    """Equal bits, any NaN like any other."""
    a, b = a.contiguous(), b.contiguous()
    if a.is_floating_point():
        nan_a, nan_b = torch.isnan(a.float()), torch.isnan(b.float())
        return bool((nan_a == nan_b).all()) and bool((_bits(a)[~nan_a] == _bits(b)[~nan_b]).all())
    return torch.equal(a, b)


class Pool:
    """Pages of NaN (or codes with NaN scales), a table of them in another order than the sequences', on the CPU and the GPU."""

    def __init__(self, lengths, heads, D, page, cache, dtype, seed=0, spare=3, max_pages=None):
        r = np.random.default_rng(seed)
        counts = [-(-n // page) for n in lengths]
        self.P = sum(counts) + spare
        order = r.permutation(self.P)
        width = max_pages or max(1, max(counts))
        self.table = np.full((len(lengths), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.lengths, self.heads, self.D, self.page, self.cache, self.dtype = lengths, heads, D, page, cache, dtype
        t = TYPES[cache]
        shape = (self.P, heads, page, D)
        if cache in oracle.LARGEST:
            # (codes that are no places hold what e4m3 has for NaN)
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8).view(t) for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:3], float("nan")) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=t) for _ in range(2))
            self.ks = self.vs = None

    def put(self, b, pos, k, v):
        """Rows [heads, D] float32 (already of dtype's values) to a place: what they stand for afterwards, float64 (None: no place)."""
        at = oracle.place(b, pos, self.table, self.page, self.P)
        if at is None:
            return None
        got = []
        for pages, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            if scales is None:
                pages[at[0], :, at[1]] = torch.from_numpy(x).to(pages.dtype)
                got.append(x.astype(np.float64))
                continue
            rows = []
            for h in range(self.heads):
                code, scale = oracle.encode(x[h], self.cache)
                pages[at[0], h, at[1]] = torch.from_numpy(code).float().to(pages.dtype)
                scales[at[0], h, at[1]] = float(scale)
                rows.append(code * float(scale))
            got.append(np.array(rows))
        return got

    def device(self):
        cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
        return lib.DeviceKvCache(cuda(self.k), cuda(self.v), cuda(self.ks), cuda(self.vs), dtype=self.dtype)

    def same(self, cache):
        assert _same_bits(cache.k_pages.cpu(), self.k) and _same_bits(cache.v_pages.cpu(), self.v)
        if self.ks is not None:
            assert _same_bits(cache.k_scales.cpu(), self.ks) and _same_bits(cache.v_scales.cpu(), self.vs)


def _values(r, shape, dtype):
    """Values of dtype as float32, rows of different sizes."""
    x = r.normal(size=shape) * np.exp(r.normal(size=shape[:-1] + (1,)))
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])


CACHES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "int8"), ("f32", "int8"), ("bf16", "e4m3"), ("f32", "e4m3")]


@pytest.mark.parametrize("dtype, cache", CACHES)
@pytest.mark.parametrize("heads, D, page, N", [(1, 16, 16, 1), (8, 64, 16, 33), (3, 80, 48, 70), (2, 128, 64, 40), (1, 256, 32, 37), (5, 48, 16, 9)])
def test_rows_into_the_cache_and_back(dtype, cache, heads, D, page, N):
    r = np.random.default_rng(N + D)
    lengths = [41, 1, page, 2 * page + 1]
    pool = Pool(lengths, heads, D, page, cache, dtype, seed=D)
    pool.table[3, 1] = r.choice([-1, pool.P, 2 ** 31 - 1, -2 ** 31])      # no page in the middle of a sequence
    c = pool.device()
    cells = [(b, i) for b, n in enumerate(lengths) for i in range(n)]
    places = [cells[i] for i in r.permutation(len(cells))[:N]]
    odd = [(-1, 3), (4, 0), (0, -1), (0, 2 ** 31 - 1), (2 ** 31 - 1, 0), (1, pool.table.shape[1] * page)]
    where = places + odd
    where = [where[i] for i in r.permutation(len(where))]
    # parts of a wider projection; rows of no place hold NaN
    wide = _values(r, (len(where), 2 * heads + 1, D), dtype)
    for n, (b, p) in enumerate(where):
        if oracle.place(b, p, pool.table, page, pool.P) is None:
            wide[n] = float("nan")
    seq, pos = (torch.tensor([w[i] for w in where], dtype=torch.int32) for i in (0, 1))
    table = torch.from_numpy(pool.table).cuda()
    on = wide.cuda()
    c.write(on[:, :heads], on[:, heads:2 * heads], seq.cuda(), pos.cuda(), table)
    held = [pool.put(b, p, wide[n, :heads].float().numpy(), wide[n, heads:2 * heads].float().numpy()) for n, (b, p) in enumerate(where)]
    pool.same(c)
    kb, k = _guarded((len(where), heads, D), TYPES[dtype])
    vb, v = _guarded((len(where), heads, D), TYPES[dtype])
    c.read(seq.cuda(), pos.cuda(), table, k, v)
    for i, x in enumerate((k, v)):
        want = torch.from_numpy(np.array([np.zeros((heads, D)) if w is None else w[i] for w in held]))
        want = want.float() if cache in oracle.LARGEST else want      # (a code times its scale, rounded to float, then to dtype)
        assert _same_bits(x.cpu(), want.to(TYPES[dtype]))
    for b in (kb, vb):
        assert (b[-GUARD:].float() == 7.0).all()
    pool.same(c)


@pytest.mark.parametrize("dtype, cache", [c for c in CACHES if c[1] in oracle.LARGEST])
def test_codes_of_every_size_of_value(dtype, cache):
    """Ties, the smallest and largest floats, rows of zeros, of infinities and NaN."""
    D, heads, N = 64, 1, 600
    r = np.random.default_rng(5)
    x = r.normal(size=(N, D)) * 2.0 ** r.integers(-20, 20, (N, 1))
    x[:100] = r.integers(-127, 128, (100, D)) / 2.0                          # ties of int8 codes
    x[:100, 0] = 127.0
    x[100:200] = r.integers(-2 ** 8, 2 ** 8, (100, D)) * 2.0 ** r.integers(-12, 1, (100, D))      # ties of e4m3 codes
    x[100:200, 0] = 448.0
    x[200:300] *= 2.0 ** r.integers(-25, 0, (100, D))
    x = x.astype(np.float32)
    x[300] = 0
    x[301] = 1e-38
    x[302] = 1e-45
    x[303] = 2.0 ** -113
    x[304] = 3e38
    x[305, 3] = np.inf
    x[306, 63] = np.nan
    x[307, 0], x[307, 1] = -np.inf, np.nan
    x = torch.from_numpy(x).to(TYPES[dtype])
    pool = Pool([N], heads, D, 16, cache, dtype)
    c = pool.device()
    rows = x.view(N, 1, D).cuda()
    seq, pos = torch.zeros(N, dtype=torch.int32, device="cuda"), torch.arange(N, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(pool.table).cuda()
    c.write(rows, -rows, seq, pos, table)
    held = [pool.put(0, n, x[n:n + 1].float().numpy(), -x[n:n + 1].float().numpy()) for n in range(N)]
    pool.same(c)
    k, v = c.read(seq, pos, table)
    for got, i in ((k, 0), (v, 1)):
        assert _same_bits(got.cpu(), torch.from_numpy(np.array([h[i] for h in held])).float().to(TYPES[dtype]))
    assert torch.isnan(k[305:308].float()).all()
    finite = x.float().numpy()[:305]
    off = np.abs(k.float().cpu().numpy()[:305, 0] - finite)
    top = np.abs(finite).max(axis=1, keepdims=True)
    half = top / 254 if cache == "int8" else np.maximum(np.abs(finite) * 2.0 ** -4, top * 2.0 ** -10 / 448)
    tiny = 2.0 ** -121 if cache == "int8" else 2.0 ** -130     # (half a code of the smallest scale)
    near = finite if dtype == "f32" else k.float().cpu().numpy()[:305, 0]
    assert (off <= half * (1 + 2.0 ** -20) + tiny + (np.abs(near) * BF if dtype == "bf16" else 0)).all()


class Attn:
    def __init__(self, lengths, T, heads, G, D, page, dtype, cache, window=0, scale=None, seed=0, max_len=None, table_width=None, bad=0.0):
        r = np.random.default_rng(seed + 17 * len(lengths))
        self.T, self.heads, self.G, self.D, self.window, self.dtype, self.cache = T, heads, G, D, window, dtype, cache
        self.scale = D ** -0.5 if scale is None else scale
        self.lengths = lengths
        self.max_len = max_len or max(1, max(lengths))
        self.pool = Pool(lengths, heads, D, page, cache, dtype, seed, max_pages=table_width or -(-self.max_len // page))
        t = self.pool.table
        hit = (r.uniform(size=t.shape) < bad) & (t >= 0)
        t[hit] = r.choice([-1, self.pool.P, 2 ** 30, -2 ** 31], size=int(hit.sum()))
        self.k, self.v, self.there = [], [], []
        for b, n in enumerate(lengths):
            ks, vs, there = np.zeros((n, heads, D)), np.zeros((n, heads, D)), np.zeros(n, dtype=bool)
            for i in range(n):
                x = _values(r, (2, heads, D), dtype).float().numpy()
                got = self.pool.put(b, i, x[0], x[1])
                if got is not None:
                    ks[i], vs[i], there[i] = got[0], got[1], True
            self.k.append(ks)
            self.v.append(vs)
            self.there.append(there)
        wide = torch.from_numpy(r.normal(size=(len(lengths), T, heads * G + 1, D)).astype(np.float32) * 1.5).to(TYPES[dtype])
        self.q64 = wide[:, :, :heads * G].double().numpy()
        self.q = wide.cuda()[:, :, :heads * G]
        self.c = self.pool.device()
        self.table = torch.from_numpy(self.pool.table).cuda()
        self.len_d = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.h = lib.DeviceKvAttn(self.c, len(lengths), T, heads * G, self.max_len, window=window, scale=scale)

    def run(self):
        self.ob, self.out = _guarded((len(self.lengths), self.T, self.heads * self.G, self.D), TYPES[self.dtype])
        self.lb, self.lse = _guarded((len(self.lengths), self.T, self.heads * self.G), torch.float32)
        self.h.fwd(self.q, self.table, self.len_d, self.out, self.lse)
        return self

    def want(self):
        """(out, its bound, lse, its bound)."""
        got = []
        for b, n in enumerate(self.lengths):
            k, v, q = self.k[b], self.v[b], self.q64[b]
            o, lse = oracle.attn(q, k, v, self.there[b], self.scale, self.window)
            mag, _ = oracle.attn(q, k, np.abs(v), self.there[b], self.scale, self.window)
            bo, bl = np.zeros(o.shape), np.zeros(lse.shape)
            for t in range(self.T):
                pos = n - self.T + t
                if pos < 0:
                    continue
                for h in range(self.heads * self.G):
                    kk = k[:pos + 1, h // self.G][self.there[b][:pos + 1]]
                    if not len(kk):
                        continue
                    s = self.scale * (kk @ q[t, h])
                    ds = (2 * (self.D + 8) * U * abs(self.scale) * (np.abs(kk) @ np.abs(q[t, h])) + 8 * U * np.abs(s)).max()
                    spread = np.abs(s).max() * 2
                    rel = 2 * ds + 2 * (6 + spread) * U + 4 * (len(kk) + 8) * U + (2.0 ** -16 if self.dtype == "bf16" else 2.0 ** -22)
                    bo[t, h] = rel * mag[t, h] + (BF if self.dtype == "bf16" else 0) * (np.abs(o[t, h]) + rel * mag[t, h])
                    bl[t, h] = ds + (6 + spread + 2 * (len(kk) + 8)) * U + np.abs(lse[t, h]) * 4 * U
            got.append((o, bo, lse, bl))
        return [np.array(x) for x in zip(*got)]

    def check(self):
        o, bo, lse, bl = self.want()
        out, got_lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        empty = np.isneginf(lse)
        assert (np.isneginf(got_lse) == empty).all() and np.isfinite(got_lse[~empty]).all() and np.isfinite(out).all()
        assert not out[empty].any()
        over = np.abs(out - o) - bo - 1e-36
        assert (over <= 0).all(), f"out: off by {np.abs(out - o).flat[over.argmax()]:.3g}, bound {bo.flat[over.argmax()]:.3g}"
        over = np.abs(got_lse[~empty] - lse[~empty]) - bl[~empty]
        assert (over <= 0).all(), f"lse: over its bound by {over.max():.3g}"
        for b in (self.ob, self.lb):
            assert (b[-GUARD:].float() == 7.0).all()
        return self


@pytest.mark.parametrize("dtype, cache", CACHES)
@pytest.mark.parametrize("lengths, T, heads, G, D, page, window", [
    ([1], 1, 1, 1, 16, 16, 0), ([0, 5, 16, 17], 1, 2, 1, 32, 16, 0), ([33, 0, 130, 64], 1, 2, 3, 64, 32, 0), ([100, 1, 47], 4, 1, 4, 80, 48, 0),
    ([513, 7, 1100], 1, 2, 4, 128, 64, 0), ([700, 3, 650], 5, 1, 8, 96, 16, 100), ([40, 200], 1, 3, 5, 256, 16, 0), ([300, 90], 9, 2, 8, 48, 32, 7),
    ([260, 31], 3, 1, 17, 192, 16, 0), ([129], 64, 1, 2, 64, 16, 0), ([900, 20], 2, 4, 2, 64, 128, 1)])
def test_attention(dtype, cache, lengths, T, heads, G, D, page, window):
    Attn(lengths, T, heads, G, D, page, dtype, cache, window, seed=D + T).run().check()
