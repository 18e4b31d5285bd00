"""The oracle of serving word by word (cache, attention over it, verification) by what its equations fix, and the library's
refusals, without a GPU."""
import itertools
import os
import re

import numpy as np
import pytest

import paper_1909_00562_amd as lib
from oracle import serving_oracle as oracle
from paper_1909_00562_amd import binding as bd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- codes ---------------------------------------------------------------------------------------------------------------


def test_codes_are_those_of_the_type():
    """The 8-bit float's values as torch has them; every code is its own code; what lies between two goes to the nearer, ties to even."""
    torch = pytest.importorskip("torch")
    bits = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    values = bits.view(torch.float8_e4m3fn).float().numpy()
    values = np.unique(values[np.isfinite(values)])
    x = np.concatenate([values, (values[1:] + values[:-1]) / 2, values[1:] * 0.9 + values[:-1] * 0.1]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    code, scale = oracle.encode(np.concatenate([[448.0], x]), "e4m3")
    assert scale == 1.0
    assert (code[1:] == torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()).all()
    x = np.arange(-254, 255) / 2
    code, scale = oracle.encode(np.concatenate([[127.0], x]), "int8")
    assert scale == 1.0 and (code[1:] == np.rint(x)).all()


@pytest.mark.parametrize("cache", ["int8", "e4m3"])
def test_codes_are_near_what_they_stand_for(cache):
    r = np.random.default_rng(1)
    for _ in range(50):
        x = (r.normal(size=64) * 2.0 ** r.integers(-60, 60)).astype(np.float32)
        code, scale = oracle.encode(x, cache)
        top = float(np.abs(x).max())
        half = top / 254 if cache == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, top / 448 * 2.0 ** -10)
        assert (np.abs(code * float(scale) - x) <= half * (1 + 2.0 ** -20)).all()
        assert np.abs(code).max() == oracle.LARGEST[cache]
    code, scale = oracle.encode(np.zeros(16), cache)
    assert not code.any() and scale == 2.0 ** -120
    for bad in (np.nan, np.inf, -np.inf):
        code, scale = oracle.encode([1.0, bad], cache)
        assert not code.any() and np.isnan(scale)


def test_places():
    table = np.array([[3, -1, 9], [2, 4, 0]])
    assert oracle.place(0, 5, table, 16, 9) == (3, 5) and oracle.place(1, 47, table, 16, 9) == (0, 15)
    for seq, pos in ((0, 16), (0, 32), (-1, 0), (2, 0), (0, -1), (1, 48)):
        assert oracle.place(seq, pos, table, 16, 9) is None


# ---- attention -----------------------------------------------------------------------------------------------------------


def _states(n, T=2, heads=2, G=2, D=4, seed=0):
    r = np.random.default_rng(seed)
    return r.normal(size=(T, heads * G, D)), r.normal(size=(n, heads, D)), r.normal(size=(n, heads, D)), np.ones(n, dtype=bool)


def test_one_token_is_attended_to_alone():
    q, k, v, there = _states(1, T=1)
    out, lse = oracle.attn(q, k, v, there, 0.7)
    for h in range(4):
        assert np.allclose(out[0, h], v[0, h // 2]) and np.isclose(lse[0, h], 0.7 * q[0, h] @ k[0, h // 2])


def test_attention_does_not_see_ahead_nor_behind_the_window():
    q, k, v, there = _states(9, T=3)
    out, lse = oracle.attn(q, k, v, there, 0.5, window=4)
    for t in range(3):
        end = 9 - 3 + t + 1
        one, lse_one = oracle.attn(q[t:t + 1], k[end - 4:end], v[end - 4:end], there[:4], 0.5)
        assert np.allclose(out[t], one[0]) and np.allclose(lse[t], lse_one[0])
    first, _ = oracle.attn(q, k[:2], v[:2], there[:2], 0.5)       # the first token's position is -1
    assert not first[0].any() and first[1].any()


def test_uniform_scores_average_and_missing_tokens_count_for_nothing():
    q, k, v, there = _states(6, T=1)
    out, lse = oracle.attn(q * 0, k, v, there, 1.0)
    assert np.allclose(out[0, 0], v[:, 0].mean(axis=0)) and np.allclose(lse, np.log(6))
    there[[1, 4]] = False
    k[[1, 4]] = np.nan
    v[[1, 4]] = np.inf
    out, lse = oracle.attn(q, k, v, there, 1.0)
    keep = [0, 2, 3, 5]
    again, lse2 = oracle.attn(q, k[keep], v[keep], np.ones(4, dtype=bool), 1.0)
    assert np.allclose(out, again) and np.allclose(lse, lse2)
    out, lse = oracle.attn(q, k, v, np.zeros(6, dtype=bool), 1.0)
    assert not out.any() and np.isneginf(lse).all()


def test_attention_of_two_parts_joins_by_their_sums():
    q, k, v, there = _states(11, T=1)
    out, lse = oracle.attn(q, k, v, there, 1.0)
    a, la = oracle.attn(q, k[:4], v[:4], there[:4], 1.0)
    b, lb = oracle.attn(q, k[4:], v[4:], there[4:], 1.0)
    assert np.allclose(lse, np.logaddexp(la, lb))
    assert np.allclose(out, a * np.exp(la - lse)[..., None] + b * np.exp(lb - lse)[..., None])


# ---- verification --------------------------------------------------------------------------------------------------------


def test_words_are_distributed_as_the_target_says():
    """The sum over what is drafted and the integral over both random numbers, on a grid: min(p, q) accepted, and p in all.
    (48 cells have the borders 1/4, of acceptance, and 2/3, between the words that are left, at their edges.)"""
    p, q = np.array([0.5, 0.125, 0.25, 0.125]), np.array([0.25, 0.5, 0.125, 0.125])
    t, d = np.log(p)[None].repeat(2, axis=0), np.log(q)[None]
    grid = (np.arange(48) + 0.5) / 48
    got, accepted = np.zeros(4), 0.0
    for x, u, w in itertools.product(range(4), grid, grid):
        n, words = oracle.verify(t, d, [x], [u], w, 1.0)
        got[words[0]] += q[x] / 48 ** 2
        accepted += n * q[x] / 48 ** 2
    assert np.allclose(got, p) and np.isclose(accepted, np.minimum(p, q).sum())


def test_a_draft_that_agrees_is_accepted_and_an_impossible_one_is_not():
    r = np.random.default_rng(0)
    t = r.normal(size=(4, 20))
    n, words = oracle.verify(t, t[:3], [3, 5, 7], [0.999] * 3, 0.5, 0.8)
    assert n == 3 and list(words[:3]) == [3, 5, 7] and words[3] >= 0
    t[1, 5] = -np.inf
    n, words = oracle.verify(t, np.zeros((3, 20)), [3, 5, 7], [0.0] * 3, 0.5, 1.0)
    assert n == 1 and words[1] not in (-1, 5) and (words[2:] == -1).all()
    n, words = oracle.verify(t, t[:3], [3, -1, 7], [0.0] * 3, 0.0, 1.0)
    assert n == 1 and words[1] == 0
    t[1, 2] = np.nan
    n, words = oracle.verify(t, t[:3], [3, 5, 7], [0.0] * 3, 0.0, 1.0)
    assert n == 0 or (n == 1 and (words[1:] == -1).all())


# ---- the library ---------------------------------------------------------------------------------------------------------


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "kv_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(kv_cache_\w+)\s*\(", text))
    assert names == set(bd.KV_EXPORTS)
    handle = lib.load_library()
    for n in names:
        assert getattr(handle, n) is not None


# fake, 16-byte aligned, never dereferenced addresses: every check fails before a launch
A = [0x10000 * (i + 1) for i in range(16)]


def _cache(**kw):
    d = dict(pages=9, page=16, heads=2, D=32, dtype=bd.AS_BF16, cache_type=bd.KC_INT8, B=3, max_pages=4)
    d.update(kw)
    return bd.KcCache(*d.values())


def _attn(**kw):
    d = dict(T=2, q_heads=4, max_len=64, window=0, scale=0.5)
    d.update(kw)
    return bd.KcAttn(*d.values())


BAD_CACHES = [(dict(pages=0), 2), (dict(page=0), 2), (dict(page=24), 2), (dict(page=8192), 2), (dict(pages=1 << 27), 2), (dict(heads=0), 2),
              (dict(heads=1025), 2), (dict(D=8), 2), (dict(D=40), 2), (dict(D=272), 2), (dict(B=0), 2), (dict(B=65537), 2), (dict(max_pages=0), 2),
              (dict(B=65536, max_pages=1 << 15), 2), (dict(max_pages=1 << 27), 2), (dict(dtype=2), 3), (dict(cache_type=4), 3),
              (dict(cache_type=bd.KC_F32), 3), (dict(dtype=bd.AS_F32, cache_type=bd.KC_BF16), 3)]


def _write(c=None, N=5, ld_k=64, ld_v=64, **kw):
    p = dict(k=A[0], v=A[1], seq=A[2], pos=A[3], table=A[4], kp=A[5], vp=A[6], ks=A[7], vs=A[8])
    p.update(kw)
    return bd.kv_cache_write(_cache() if c is None else c, N, p["k"], ld_k, p["v"], ld_v, p["seq"], p["pos"], p["table"], p["kp"], p["vp"],
                             p["ks"], p["vs"], check=False)


def _read(c=None, N=5, **kw):
    p = dict(k=A[0], v=A[1], seq=A[2], pos=A[3], table=A[4], kp=A[5], vp=A[6], ks=A[7], vs=A[8])
    p.update(kw)
    return bd.kv_cache_read(_cache() if c is None else c, N, p["kp"], p["vp"], p["ks"], p["vs"], p["seq"], p["pos"], p["table"], p["k"],
                            p["v"], check=False)


def _run(c=None, a=None, ld_q=128, ws=1 << 40, **kw):
    p = dict(q=A[0], kp=A[1], vp=A[2], ks=A[3], vs=A[4], table=A[5], lengths=A[6], out=A[7], lse=None, workspace=A[8])
    p.update(kw)
    return bd.kv_cache_attn(_cache() if c is None else c, _attn() if a is None else a, p["q"], ld_q, p["kp"], p["vp"], p["ks"], p["vs"],
                            p["table"], p["lengths"], p["out"], p["lse"], p["workspace"], ws, check=False)


@pytest.mark.parametrize("kw, code", BAD_CACHES)
def test_caches_that_are_refused(kw, code):
    c = _cache(**kw)
    assert _write(c) == code and _read(c) == code and _run(c) == code
    assert bd.kv_cache_attn_workspace_bytes(c, _attn()) == 0


def test_rows_that_are_refused():
    for f in (_write, _read):
        assert f(N=0) == 2 and f(N=(1 << 24) + 1) == 2
        for name in ("k", "v", "seq", "pos", "table", "kp", "vp", "ks", "vs"):
            assert f(**{name: None}) == 1, name
            assert f(**{name: A[9] + 4}) == 5, name
        assert f(_cache(cache_type=bd.KC_BF16)) == 1                     # scales of a cache that has none
    assert _write(vp=A[5]) == 2 and _write(vs=A[7]) == 2 and _read(vp=A[5], N=0) == 2      # (one pool for both is only read)
    assert bd.kv_cache_write(None, 5, A[0], 64, A[1], 64, *A[2:9], check=False) == 1
    for kw in (dict(ld_k=63), dict(ld_v=48), dict(ld_k=-64), dict(ld_v=1 << 32)):
        assert _write(**kw) == 2, kw
    assert _write(ld_k=68) == 5 and _write(_cache(dtype=bd.AS_F32), ld_v=66) == 5


def test_attention_that_is_refused():
    assert bd.kv_cache_attn_workspace_bytes(_cache(), _attn()) >= 16
    assert bd.kv_cache_attn_workspace_bytes(_cache(max_pages=400), _attn(max_len=6400)) > 16
    for kw in (dict(T=0), dict(T=65), dict(q_heads=0), dict(q_heads=3), dict(T=64, q_heads=34), dict(max_len=0), dict(max_len=65), dict(window=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-3e38)):
        assert _run(a=_attn(**kw)) == 2, kw
        assert bd.kv_cache_attn_workspace_bytes(_cache(), _attn(**kw)) == 0, kw
    for name in ("q", "kp", "vp", "ks", "vs", "table", "lengths", "out", "workspace"):
        assert _run(**{name: None}) == 1, name
    for name in ("q", "kp", "vp", "ks", "vs", "table", "lengths", "out", "lse", "workspace"):
        assert _run(**{name: A[9] + 4}) == 5, name
    assert _run(ld_q=127) == 2 and _run(ld_q=132) == 5 and _run(ws=15) == 4
    assert "needed" in bd.attn_softmax_last_error()
    # 2^16 sequences of 1024 heads and 2^20 tokens are more chunks than are counted
    big = _cache(B=65536, heads=1024, max_pages=1 << 9, page=2048)
    assert _run(big, _attn(q_heads=1024, max_len=1 << 20), ld_q=1 << 20) == 2
    many = _cache(B=65536, heads=65, max_pages=1)                            # 65536 x 65 blocks of 512 threads
    assert _run(many, _attn(T=1, q_heads=65, max_len=16), ld_q=1 << 16) == 2
    assert bd.kv_cache_attn_workspace_bytes(_cache(B=65536, heads=64, max_pages=1), _attn(T=1, q_heads=64, max_len=16)) > 0
    assert bd.kv_cache_attn_workspace_bytes(_cache(max_pages=1 << 24), _attn(max_len=(1 << 28) - 1)) > 0
    assert bd.kv_cache_attn_workspace_bytes(_cache(max_pages=1 << 24), _attn(max_len=1 << 28)) == 0
    assert bd.kv_cache_attn_workspace_bytes(_cache(), _attn(window=2 ** 31 - 1)) > 0


def test_verification_that_is_refused():
    def shape(**kw):
        d = dict(B=2, T=3, V=100, dtype=bd.AS_F32, temperature=1.0)
        d.update(kw)
        return bd.VoVerify(*d.values())

    def run(s, ld_t=100, ld_d=100, ws=1 << 40, **kw):
        p = dict(target=A[0], draft=A[1], drafted=A[2], u=A[3], un=A[4], n=A[5], words=A[6], workspace=A[7])
        p.update(kw)
        return bd.vocab_verify(s, p["target"], ld_t, p["draft"], ld_d, p["drafted"], p["u"], p["un"], p["n"], p["words"], p["workspace"], ws, check=False)

    assert bd.vocab_verify_workspace_bytes(shape()) > 0
    for kw, code in ((dict(B=0), 2), (dict(B=65537), 2), (dict(T=0), 2), (dict(T=65), 2), (dict(V=0), 2), (dict(V=(1 << 20) + 1), 2), (dict(dtype=2), 3),
                     (dict(temperature=0.0), 2), (dict(temperature=2.0 ** -11), 2), (dict(temperature=2000.0), 2), (dict(temperature=float("nan")), 2)):
        assert run(shape(**kw)) == code, kw
        assert bd.vocab_verify_workspace_bytes(shape(**kw)) == 0
    assert run(None) == 1
    for name in ("target", "draft", "drafted", "u", "un", "n", "words", "workspace"):
        assert run(shape(), **{name: None}) == 1, name
        assert run(shape(), **{name: A[9] + 4}) == 5, name
    assert run(shape(), ld_t=99) == 2 and run(shape(), ld_d=96) == 2 and run(shape(), ld_t=102) == 5
    assert run(shape(dtype=bd.AS_BF16), ld_t=104, ld_d=108) == 5 and run(shape(), ws=100) == 4


def test_handles_need_a_gpu():
    torch = pytest.importorskip("torch")
    pages = torch.zeros(2, 1, 16, 16)
    for make in (lambda: lib.DeviceKvCache(pages, pages), lambda: lib.DeviceVocabVerify(1, 1, 16, device="cpu")):
        with pytest.raises(bd.AttnSoftmaxError) as e:
            make()
        assert e.value.code == 2
