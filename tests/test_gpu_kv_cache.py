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


@pytest.mark.parametrize("dtype, cache", CACHES)
def test_attention_of_most_rows_and_most_heads(dtype, cache):
    Attn([90, 64], 64, 1, 16, 16, 4096, dtype, cache, seed=17).run().check()
    Attn([18, 0, 1], 1, 1024, 1, 16, 16, dtype, cache, seed=18).run().check()


@pytest.mark.parametrize("dtype, cache", CACHES)
def test_attention_past_pages_that_are_none(dtype, cache):
    """Tokens whose page is none are not seen; sequences of none give zeros; what is behind the end, and pages that nobody names, hold NaN."""
    Attn([700, 90, 33, 1], 2, 2, 2, 64, 16, dtype, cache, seed=3, bad=0.4).run().check()
    c = Attn([64, 40], 1, 1, 3, 48, 16, dtype, cache, seed=4)
    c.table[1] = -1
    c.run()
    assert not c.out[1].any() and torch.isneginf(c.lse[1]).all()
    c.there[1][:] = False
    c.check()
    Attn([500, 2000], 3, 2, 2, 64, 48, dtype, cache, window=900, seed=5, bad=0.2, table_width=60).run().check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype, cache", [c for c in CACHES if c[1] != "int8"])
@pytest.mark.parametrize("D", [48, 128, 256])
def test_values_that_a_row_does_not_see_do_not_reach_it(dtype, cache, D, bad):
    """Infinities and NaN in the cache at tokens that some rows see and others do not: the end of a draft, the beginning of a window, and
    in one column and one head alone."""
    lengths, T, window, col = [200, 37, 100], 6, 31, 7
    c = Attn(lengths, T, 2, 3, D, 16, dtype, cache, window=window, seed=6)
    o, bo, lse, bl = c.want()
    v = c.c.v_pages
    odd = []                                                  # (sequence, token)
    for b, n in enumerate(lengths):
        odd += [(b, n - 2), (b, n - T - window + 2), (b, max(0, n - T - window - 1))]
    for b, i in odd:
        if i < 0:
            continue
        p, at = oracle.place(b, i, c.pool.table, 16, c.pool.P)
        if cache == "e4m3":
            if bad == bad:
                return                                        # (the type has no infinity)
            v.view(torch.uint8)[p, 1, at, col] = 0x7f
        else:
            v[p, 1, at, col] = bad
    c.run()
    out = c.out.double().cpu().numpy()
    for b, n in enumerate(lengths):
        for t in range(T):
            pos = n - T + t
            sees = [i for x, i in odd if x == b and 0 <= i <= pos and i > pos - window]
            hit = np.zeros((6, D), dtype=bool)
            if sees:
                hit[3:, col] = True                           # the heads that read head 1
            assert not np.isfinite(out[b, t][hit]).any()
            assert (np.abs(out[b, t] - o[b, t])[~hit] <= bo[b, t][~hit] + 1e-36).all()
    assert np.isfinite(c.lse.cpu().numpy()[~np.isneginf(lse)]).all()


@pytest.mark.parametrize("dtype, cache", CACHES)
def test_keys_that_are_no_numbers(dtype, cache):
    """A NaN in a seen key makes its rows NaN, and those of other heads and sequences are as they were."""
    c = Attn([300, 80], 2, 2, 2, 64, 16, dtype, cache, seed=7)
    o, bo, _, _ = c.want()
    p, at = oracle.place(0, 299, c.pool.table, 16, c.pool.P)      # the last token: seen by the second row alone
    if cache in oracle.LARGEST:
        c.c.k_scales[p, 0, at] = float("nan")
    else:
        c.c.k_pages[p, 0, at, 5] = float("nan")
    c.run()
    out, lse = c.out.double().cpu().numpy(), c.lse.cpu().numpy()
    assert np.isnan(out[0, 1, :2]).all() and np.isnan(lse[0, 1, :2]).all()
    out[0, 1, :2] = o[0, 1, :2]
    assert (np.abs(out - o) <= bo + 1e-36).all()


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0])
@pytest.mark.parametrize("dtype, cache", CACHES)
def test_scales_of_any_sign(dtype, cache, scale):
    Attn([130, 5], 2, 1, 2, 32, 16, dtype, cache, scale=scale, seed=8).run().check()


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "int8")])
@pytest.mark.parametrize("order", ["up", "down"])
def test_scores_that_grow_and_shrink(dtype, cache, order):
    """Maxima that move at every step, by less and by more than what the running one may lag behind: keys in the order of their scores,
    over powers of two from 2^-60 to 2^60 of weight."""
    c = Attn([900], 1, 1, 1, 16, 16, dtype, cache, scale=1.0, seed=9)
    rows = np.zeros((900, 1, 16), dtype=np.float32)
    ramp = np.linspace(-42, 42, 900)
    rows[:, 0, 0] = torch.from_numpy(ramp if order == "up" else ramp[::-1].copy()).to(TYPES[dtype]).float().numpy()
    for i in range(900):
        got = c.pool.put(0, i, rows[i], c.v[0][i].astype(np.float32) if cache not in oracle.LARGEST else rows[i] * 0.1 + 1)
        c.k[0][i], c.v[0][i] = got
    c.c = c.pool.device()
    c.h = lib.DeviceKvAttn(c.c, 1, 1, 1, 900, scale=1.0)
    q = torch.zeros(1, 1, 1, 16)
    q[..., 0] = 1
    c.q, c.q64 = q.to(TYPES[dtype]).cuda(), q.double().numpy()
    c.run().check()


def test_keys_and_values_in_one_pool_and_shared_pages():
    c = Attn([100, 100], 1, 2, 2, 64, 16, "bf16", "bf16", seed=10)
    one = lib.DeviceKvCache(c.c.k_pages, c.c.k_pages)
    c.h = lib.DeviceKvAttn(one, 2, 1, 4, 100)
    c.v = c.k
    c.run().check()
    # the second sequence begins with the first one's pages
    c.table[1, :4] = c.table[0, :4]
    c.k[1][:64] = c.k[0][:64]
    c.run().check()


def _in_64_bits(c, b, h):
    """out and lse of a sequence's head of queries on the GPU, T = 1; and magnitudes, for its bound."""
    n, kv = c["lengths"][b], h // c["G"]
    ids = c["table"][b, :-(-n // c["page"])].long()
    rows = []
    for pages, scales in ((c["c"].k_pages, c["c"].k_scales), (c["c"].v_pages, c["c"].v_scales)):
        x = pages.view(torch.uint8)[ids, kv].view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else pages[ids, kv]
        x = x.double()
        if scales is not None:
            x = x * scales[ids, kv].double()[..., None]
        rows.append(x.reshape(-1, pages.shape[3])[:n])
    q = c["q"][b, 0, h].double()
    s = rows[0] @ q * c["scale"]
    w = torch.softmax(s, 0)
    mag = rows[0].abs() @ q.abs() * c["scale"]
    return w @ rows[1], torch.logsumexp(s, 0), w @ rows[1].abs(), float(mag.max()), float(s.abs().max())


# Long sequences, many of them, offsets past 32 bits: a pool of 5 GB in bf16.  Against float64 on the GPU, some heads of each.
@pytest.mark.parametrize("lengths, heads, G, D, page, dtype, cache, spread", [
    ([131071, 3, 70000], 2, 4, 128, 128, "bf16", "int8", 1), ([40000, 39999], 8, 1, 64, 16, "f32", "f32", 1), ([9000] * 40, 4, 8, 128, 64, "bf16", "bf16", 1),
    (list(range(1, 601)), 2, 2, 32, 16, "bf16", "e4m3", 1), ([5000, 60000], 8, 2, 128, 64, "bf16", "bf16", 36)])
def test_attention_of_long_sequences(lengths, heads, G, D, page, dtype, cache, spread):
    gen = torch.Generator(device="cuda").manual_seed(1)
    counts = [-(-n // page) for n in lengths]
    P = sum(counts) * spread
    ids = torch.randperm(P, device="cuda", generator=gen)[:sum(counts)].to(torch.int32)
    ids[-1] = P - 1 if not (ids == P - 1).any() else ids[-1]
    table = torch.full((len(lengths), max(counts)), -1, device="cuda", dtype=torch.int32)
    for b, part in enumerate(ids.split(counts)):
        table[b, :len(part)] = part
    t = TYPES[cache]
    make = lambda: torch.randn(P, heads, page, D, device="cuda", generator=gen) * 1.3  # noqa: E731
    if cache in oracle.LARGEST:
        codes = lambda: (make() * 40).clamp(-127, 127).to(t)  # noqa: E731
        scales = lambda: torch.rand(P, heads, page, device="cuda", generator=gen) * 0.03 + 0.01  # noqa: E731
        c = lib.DeviceKvCache(codes(), codes(), scales(), scales(), dtype=dtype)
    else:
        pages = []
        for _ in range(2):
            x = torch.empty(P, heads, page, D, device="cuda", dtype=t)
            for part in x.split(4096):
                part.normal_(generator=gen)
            pages.append(x)
        c = lib.DeviceKvCache(*pages)
    q = torch.randn(len(lengths), 1, heads * G, D, device="cuda", generator=gen).to(TYPES[dtype])
    h = lib.DeviceKvAttn(c, len(lengths), 1, heads * G, max(lengths))
    lse = torch.empty(len(lengths), 1, heads * G, device="cuda")
    out = h.fwd(q, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), lse=lse)
    what = dict(lengths=lengths, G=G, page=page, table=table, c=c, q=q, scale=D ** -0.5)
    for b in (range(len(lengths)) if len(lengths) < 10 else range(0, len(lengths), len(lengths) // 9)):
        for head in (0, heads * G - 1):
            o, l, mag, qk, top = _in_64_bits(what, b, head)
            # weights' errors are independent of each other's sign, but count in full here; sums of n: in runs of 32 and of a wave's steps
            n = lengths[b]
            ds = 2 * (D + 8) * U * qk + 8 * U * top
            rel = 2 * ds + 2 * (6 + 2 * top) * U + 4 * (n / 8 + 64) * U + (2.0 ** -16 if dtype == "bf16" else 2.0 ** -22)
            bound = rel * mag + (BF if dtype == "bf16" else 0) * (o.abs() + rel * mag)
            assert ((out[b, 0, head].double() - o).abs() <= bound).all(), (b, head)
            assert abs(float(lse[b, 0, head]) - float(l)) <= ds + (6 + 2 * top + 2 * (n / 8 + 64)) * U + abs(float(l)) * 4 * U


def test_long_lists_of_rows_and_offsets_past_32_bits():
    """More rows than fit the launch one after the other, and a pool of 5 GB."""
    heads, page, D = 4, 64, 128
    P = 5 * 2 ** 30 // (heads * page * D * 2)
    pages = torch.zeros(P, heads, page, D, device="cuda", dtype=torch.bfloat16)
    c = lib.DeviceKvCache(pages, torch.zeros_like(pages))
    N = 300000
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randperm(P, device="cuda", generator=gen).to(torch.int32)[None]
    pos = torch.randperm(P * page, device="cuda", generator=gen)[:N].to(torch.int32)
    pos[0] = P * page - 1
    pos = pos.unique().flip(0).contiguous()
    N = len(pos)
    seq = torch.zeros(N, dtype=torch.int32, device="cuda")
    k = torch.randn(N, heads, D, device="cuda", generator=gen).bfloat16()
    c.write(k, -k, seq, pos, table)
    got_k, got_v = c.read(seq, pos, table)
    assert torch.equal(got_k, k) and torch.equal(got_v, -k)
    at = table[0, (pos // page).long()].long()
    assert torch.equal(c.k_pages[at, :, (pos % page).long()], k)
    assert int((c.k_pages != 0).any(dim=3).sum()) <= N * heads


def test_calls_are_alike_and_captured():
    """The same bits again, on another stream, and from graphs that are replayed with eager calls between them; two graphs that share a workspace."""
    c = Attn([900, 40, 513, 1300], 2, 2, 4, 128, 64, "bf16", "int8", seed=11).run()
    out, lse = c.out.clone(), c.lse.clone()
    c.run()
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.h.fwd(c.q, c.table, c.len_d)
    side.synchronize()
    assert torch.equal(other, out)
    short = torch.tensor([90, 4, 51, 130], dtype=torch.int32, device="cuda")
    want_short = c.h.fwd(c.q, c.table, short).clone()
    graphs, outs = [], []
    for lengths in (c.len_d, short):
        o = torch.empty_like(out)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.h.fwd(c.q, c.table, lengths, o)
        graphs.append(g)
        outs.append(o)
    for _ in range(4):
        for g, o, want in zip(graphs, outs, (out, want_short)):
            o.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want)
        assert torch.equal(c.h.fwd(c.q, c.table, c.len_d), out)
    # lengths are data of the graph
    short.copy_(c.len_d)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[1], out)


def test_lengths_are_clamped():
    c = Attn([50, 64], 1, 1, 2, 32, 16, "bf16", "bf16", seed=12, max_len=64).run()
    out = c.out.clone()
    c.len_d.copy_(torch.tensor([50, 2 ** 31 - 1], dtype=torch.int32))
    assert torch.equal(c.h.fwd(c.q, c.table, c.len_d), out)
    c.len_d.copy_(torch.tensor([-5, -2 ** 31], dtype=torch.int32))
    lse = torch.empty(2, 1, 2, device="cuda")
    assert not c.h.fwd(c.q, c.table, c.len_d, lse=lse).any() and torch.isneginf(lse).all()


def test_refusals_of_the_handles():
    c = Attn([20, 30], 1, 2, 2, 32, 16, "bf16", "int8", seed=13)
    k = torch.zeros(3, 2, 32, device="cuda", dtype=torch.bfloat16)
    i = torch.zeros(3, device="cuda", dtype=torch.int32)

    def code(f):
        with pytest.raises(bd.AttnSoftmaxError) as e:
            f()
        return e.value.code

    assert code(lambda: lib.DeviceKvCache(c.c.k_pages, c.c.v_pages, c.c.k_scales, dtype="bf16")) == 1
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages, c.c.v_pages, c.c.k_scales, c.c.v_scales)) == 3
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages.half(), c.c.v_pages.half())) == 3
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages.bfloat16(), c.c.v_pages.float())) == 3
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages.bfloat16(), c.c.v_pages.bfloat16(), c.c.k_scales, c.c.v_scales)) == 1
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages.bfloat16(), c.c.v_pages.bfloat16(), dtype="f32")) == 3
    assert code(lambda: lib.DeviceKvCache(c.c.k_pages, c.c.v_pages[1:], c.c.k_scales, c.c.v_scales, dtype="bf16")) == 2
    assert code(lambda: c.c.write(k.float(), k, i, i, c.table)) == 3
    assert code(lambda: c.c.write(k[:2], k, i, i, c.table)) == 2
    assert code(lambda: c.c.write(k.transpose(0, 1).contiguous().transpose(0, 1), k, i, i, c.table)) == 5
    assert code(lambda: c.c.write(k, k, i.long(), i, c.table)) == 3
    assert code(lambda: c.c.write(k, k, i, i.cpu(), c.table)) == 2
    assert code(lambda: c.c.write(k, k, i, i, c.table[0])) == 2
    assert code(lambda: c.c.write(k, k, i, i, None)) == 1
    assert code(lambda: c.c.read(i, i, c.table, k=k.float())) == 3
    assert code(lambda: c.h.fwd(c.q, c.table, c.len_d.long())) == 3
    assert code(lambda: c.h.fwd(c.q, c.table[:, :1], c.len_d)) == 2
    assert code(lambda: c.h.fwd(c.q, c.table[:1], c.len_d)) == 2
    assert code(lambda: c.h.fwd(c.q.float(), c.table, c.len_d)) == 3
    assert code(lambda: c.h.fwd(c.q[..., :16], c.table, c.len_d)) == 2
    assert code(lambda: lib.DeviceKvAttn(c.c, 2, 1, 3, 30)) == 2
    assert code(lambda: lib.DeviceKvAttn(c.c, 2, 1, 4, 0)) == 2
    assert code(lambda: lib.DeviceKvAttn(c.c, 2, 1, 4, 30, window=-1)) == 2
    # no rows at all
    none = torch.zeros(0, device="cuda", dtype=torch.int32)
    c.c.write(k[:0], k[:0], none, none, c.table)
    assert c.c.read(none, none, c.table)[0].shape == (0, 2, 32)


# max_len far beyond the lengths: the launches of long sequences.  Up to 64 sequences a wave cuts them, beyond a block, 512 at a time; few (sequence,
# head) are cut into pieces, many into runs.
@pytest.mark.parametrize("dtype, cache, D", [("bf16", "bf16", 64), ("f32", "f32", 128), ("bf16", "e4m3", 256), ("f32", "int8", 32)])
@pytest.mark.parametrize("lengths, T, heads, G, window", [
    ([0, 1500, 0, 1], 1, 2, 2, 0), ([0, 0, 0], 2, 1, 1, 0), ([2, 600, 0, 1300, 44], 5, 1, 9, 300), ([i * 37 % 211 for i in range(70)], 1, 1, 2, 0),
    ([0] * 65 + [700, 5], 3, 1, 2, 0), ([i % 23 for i in range(600)], 1, 2, 1, 5), ([1100], 64, 1, 2, 2 ** 31 - 1)])
def test_attention_cut_into_runs_and_pieces(dtype, cache, D, lengths, T, heads, G, window):
    Attn(lengths, T, heads, G, D, 16, dtype, cache, window, seed=14, max_len=9000).run().check()


# More (sequence, head, group of rows) than runs: those that are shared are found from the runs, those that hold nothing apart.
@pytest.mark.parametrize("dtype, cache, D", [("bf16", "bf16", 64), ("f32", "f32", 128), ("f32", "e4m3", 16)])
@pytest.mark.parametrize("lengths, T, heads, G, window", [
    ([i * 5 % 9 for i in range(300)] + [400, 0, 33] + [0] * 297 + [1], 40, 3, 2, 0),       # two groups of rows to a head, the second one not full
    ([3, 0, 900, 1] + [i % 3 for i in range(56)], 1, 70, 1, 0), ([0] * 200 + [5, 700] + [2] * 3, 2, 21, 1, 0), ([0] * 130, 3, 33, 1, 4)])
def test_more_heads_than_runs(dtype, cache, D, lengths, T, heads, G, window):
    Attn(lengths, T, heads, G, D, 16, dtype, cache, window, seed=16, max_len=9000).run().check()


def test_more_blocks_than_the_chip_holds():
    """As many (sequence, head) as runs and more; long and short calls on the same cache give the same up to rounding."""
    lengths = [int(x) for x in np.random.default_rng(0).integers(0, 900, 300)]
    c = Attn(lengths, 1, 4, 2, 64, 16, "f32", "f32", seed=15)
    c.run()
    long = lib.DeviceKvAttn(c.c, 300, 1, 8, 4000)
    table = torch.full((300, 250), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    lse = torch.empty_like(c.lse)
    out = long.fwd(c.q, table, c.len_d, lse=lse)
    # two results, each within 4 (n + 24) u of the sum of weights times magnitudes (at most the largest value, here below 200)
    assert (out - c.out).abs().max() <= 2 * 4 * (900 + 24) * U * float(c.c.v_pages[~torch.isnan(c.c.v_pages)].abs().max())
    some = ~torch.isneginf(c.lse)
    assert torch.equal(torch.isneginf(lse), ~some) and (lse - c.lse)[some].abs().max() <= 1e-4
