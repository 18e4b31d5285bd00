"""The operators over the vocabulary (include/vocab_ops.h) where their errors would hide: sums that cancel, and further edges of
their range.  Against the float64 oracle, or torch in float64 for larger calls."""
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_1909_00562_amd as lib  # noqa: E402
from oracle import vocab_ops_oracle as oracle  # noqa: E402
from paper_1909_00562_amd import binding as bd  # noqa: E402
from test_gpu_vocab_ops import BF, U, Case, _in_64_bits, _round, _untouched  # noqa: E402


def _with(c, h, W, b):
    """The case with other states, weights and bias."""
    (c.h, c.h64), (c.W, c.W64), (c.b, c.b64) = (_round(x, c.dtype) for x in (h, W, b))
    c.h[~torch.from_numpy(c.word)] = float("nan")
    c.h64[~c.word] = 0.0
    return c


# A model that has learnt how often words come: W and h are mostly what their rows have in common, which cancels in dh (rows of dl sum to 0)
# and in dW (the words' probabilities are their shares of the targets).  Bound by the norm: the rounding of the result, 2^-8 of it at most, and dl
# within 2^-17 of itself, together with fp32 sums 2^-16 of the sum of magnitudes.  dl rounded once to bf16 is 1.5 to 2.1 times the bound off in dh.
@pytest.mark.parametrize("N, H, V, K", [(5, 64, 40, 0), (16, 2056, 60, 0), (12, 64, 200, 5), (40, 64, 50, 0), (300, 72, 515, 0), (700, 136, 1003, 0), (700, 136, 1003, 9), (2100, 64, 16500, 0)])
def test_bf16_gradients_where_the_sums_cancel(N, H, V, K):
    r = np.random.default_rng(N)
    y = np.clip(np.exp(r.uniform(size=N) * np.log(V)).astype(np.int64), 1, V - 1)
    c = Case(N, H, V, "bf16", "bf16", K=K, tau=2.0, targets=y, seed=N)
    mostly_common = lambda n, s: s * (6 * r.uniform(-1, 1, (1, H)) + r.uniform(-1, 1, (n, H)))  # noqa: E731
    often = np.bincount(y, minlength=V) + 0.02
    _with(c, mostly_common(N, 0.12), mostly_common(V, 0.05), np.log(often / often.max()))
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    o = oracle.loss(c.h64, c.W64, c.b64, c.y, c.pad_id, c.g, c.teacher)
    dl = np.abs(o["dl"])
    for k, mag in (("dh", dl @ np.abs(c.W64)), ("dW", dl.T @ np.abs(c.h64)), ("db", dl.sum(axis=0))):
        off = np.linalg.norm(c.out[k].double().cpu().numpy() - o[k])
        bound = BF * np.linalg.norm(o[k]) + 2.0 ** -16 * np.linalg.norm(mag)
        assert off <= bound, (k, off / bound)


# dW and dh in launches of their own (from 4096 positions on), dh split and, behind two rounds of its tiles, not; pieces of the vocabulary.  By the
# norm: the result's rounding, 2^-8 at most, and dl's two terms, 2^-17 of magnitudes that are less than 32 times the result.
@pytest.mark.parametrize("N, H, V, K", [(4100, 1000, 16003, 0), (4100, 1000, 48001, 6), (16384, 2048, 16001, 0)])
def test_bf16_gradients_of_many_positions(N, H, V, K):
    c = Case(N, H, V, "bf16", "bf16", K=K, tau=2.0, seed=N, g=1.0)
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    o = _in_64_bits(c, c.h_d, c.y_d)
    first = {}
    for k in ("dh", "dW", "db"):
        off = float((c.out[k].double() - o[k]).norm() / o[k].norm())
        assert off < 17 / 16 * BF, (k, off)
        assert not c.out["dh"][~torch.from_numpy(c.word).cuda()].any()
        first[k] = c.out[k].clone()
    c.bwd(v)
    assert all(torch.equal(first[k], c.out[k]) for k in first)


# Waves of 128 x 128 and 256 x 256 tiles whose rows all lie behind the last word's: they have no entries of the teacher to read.
@pytest.mark.parametrize("N, H, V, dtype, grad", [(140, 64, 20003, "bf16", "f32"), (300, 64, 65600, "bf16", "bf16"), (385, 40, 33000, "bf16", "f32"), (300, 40, 2001, "f32", "f32")])
def test_tiles_with_waves_behind_the_last_row(N, H, V, dtype, grad):
    c = Case(N, H, V, dtype, grad, K=6, tau=2.0, pad=0.0, seed=N)
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    c.check()


# A row of a word whose states hold a NaN or an infinity: its losses and the sums say so, whatever the kernels, and so do the gradients that it is
# part of; other rows keep their bits.
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("N, H, V, dtype, grad, K", [
    (20, 40, 300, "f32", "f32", 5), (20, 40, 300, "f32", "f32", 0), (14, 64, 300, "bf16", "bf16", 5), (40, 64, 500, "bf16", "bf16", 5), (200, 33, 300, "f32", "f32", 4),
    (700, 72, 4001, "bf16", "f32", 5), (700, 72, 4001, "bf16", "bf16", 0), (2100, 64, 16500, "bf16", "bf16", 5), (2100, 40, 16500, "f32", "f32", 3)])
def test_a_row_that_is_not_finite(N, H, V, dtype, grad, K, value):
    c = Case(N, H, V, dtype, grad, K=K, tau=2.0, pad=0.2, seed=N)
    at = int(np.nonzero(c.word)[0][N // 3])
    if K:
        c.ids[at], c.z[at] = np.arange(K), 0.5                        # it has entries
    names = ("tok_loss", "loss_sum", "dh", "dW", "db") + (("tok_distill", "distill_sum") if K else ("argmax",))
    v = c.device()
    got = []
    for x in (None, value):
        if x is not None:
            c.h_d[at, H // 2] = x
        c.fwd(v)
        c.bwd(v)
        got.append({k: c.out[k].clone() for k in names})
    clean, dirty = got
    for k in names:
        if k in ("loss_sum", "distill_sum", "dW", "db"):
            assert dirty[k].isnan().all(), k
            continue
        others = torch.arange(N, device="cuda") != at
        assert torch.equal(clean[k][others], dirty[k][others]), k
        if k == "argmax":
            assert 0 <= int(dirty[k][at]) < V
        else:
            assert dirty[k][at].isnan().all() and clean[k].isfinite().all(), k


# The most positions that there may be, with rows of more vectors than half a block has threads.
def _room(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip(f"{free >> 30} GiB free")


def test_embedding_of_the_most_positions():
    _room(48)
    N, I, V = 1 << 24, 516, 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.empty(V, I, device="cuda").uniform_(-1, 1, generator=gen)
    ids = torch.randint(-V // 4, V, (N,), device="cuda", dtype=torch.int32, generator=gen)
    x = lib.DeviceEmbed(table, N, pad_id=0, scale=2.0).fwd(ids)
    for at in torch.arange(N, device="cuda").split(1 << 21):
        want = torch.where((ids[at] > 0)[:, None], table[ids[at].clamp(min=0).long()] * 2, 0)       # (twice a value is exact)
        assert torch.equal(x[at], want)


def test_cross_entropy_of_the_most_positions():
    _room(130)
    N, H, V, bf = 1 << 24, 520, 8, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(2)
    W = torch.empty(V, H, device="cuda", dtype=bf).uniform_(-0.06, 0.06, generator=gen)
    h = torch.empty(N, H, device="cuda", dtype=bf).uniform_(-1, 1, generator=gen)
    y = torch.randint(-2, V, (N,), device="cuda", dtype=torch.int32, generator=gen)
    v = lib.DeviceVocabLoss(W, None, N, pad_id=0, grad_scale=1.0)
    loss, n_tok = torch.empty(1, device="cuda"), torch.empty(1, device="cuda", dtype=torch.int32)
    v.xent_fwd(h, y, loss, n_tok)
    dh, dW, db = torch.full_like(h, 7.0), torch.empty_like(W), torch.empty(V, device="cuda", dtype=bf)
    v.xent_bwd(dh, dW, db)
    assert int(n_tok) == int((y > 0).sum())
    zero = lambda *n: torch.zeros(*n, device="cuda", dtype=torch.float64)  # noqa: E731
    W64, o_dW, o_db, loss64, off = W.double(), zero(V, H), zero(V), zero(1), zero(2)
    for at in torch.arange(N, device="cuda").split(1 << 20):
        x, t, word = h[at].double(), y[at].clamp(min=0).long()[:, None], (y[at] > 0)[:, None]
        l = x @ W64.t()
        lse = torch.logsumexp(l, 1, keepdim=True)
        dl = torch.where(word, torch.exp(l - lse).scatter_add_(1, t, torch.full_like(lse, -1.0)), 0.0)
        loss64 += torch.where(word, lse - l.gather(1, t), 0.0).sum()
        o_dW += dl.t() @ x
        o_db += dl.sum(0)
        o = dl @ W64
        off += torch.stack([(dh[at].double() - o).square().sum(), o.square().sum()])
        assert not dh[at][~word[:, 0]].any()
    # norms: the results' rounding, and fp32 sums of 2^24 terms in a few hundred parts, 2^-24 sqrt(2^24) of their magnitudes at most
    assert float((off[0] / off[1]).sqrt()) < 2 * BF
    for k, got, o in (("dW", dW, o_dW), ("db", db, o_db)):
        assert float((got.double() - o).norm() / o.norm()) < 2 * BF, k
    assert abs(float(loss) - float(loss64)) < 1e-5 * float(loss64)


def test_a_handle_dropped_while_another_stream_works_on_it():
    """Its workspace is not given to others before that stream is through."""
    c = Case(40, 64, 500, "bf16", "f32", seed=7)
    a = torch.randn(8192, 8192, device="cuda")
    side = torch.cuda.Stream()
    v, e = c.device(), lib.DeviceEmbed(torch.zeros(500, 64, device="cuda"), 40)
    d = e.bwd(c.y_d, torch.zeros(40, 64, device="cuda"))             # (allocates its workspace here)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a @ a
        c.fwd(v)
        c.bwd(v)
        e.bwd(c.y_d, c.out["dh"], d)
    busy = {(w.data_ptr(), w.numel()) for w in (v.workspace, e.workspace)}
    del v, e
    others = [torch.empty(n, dtype=torch.uint8, device="cuda") for _, n in busy for _ in range(4)]
    assert not side.query(), "the stream was through too early to tell"
    assert not {t.data_ptr() for t in others} & {p for p, _ in busy}
    torch.cuda.synchronize()
    c.check()


# ---- pieces of the vocabulary ----------------------------------------------------------------------------------------------
# What a piece may take is a constant of vocab.hip: the cases below stay several pieces when it changes, or say so.
def _piece_bytes():
    text = open(os.path.join(os.path.dirname(bd.library_path()), "csrc", "vocab.hip")).read()
    n, shift = re.search(r"constexpr int64_t kPieceBytes = \(int64_t\)(\d+) << (\d+);", text).groups()
    return int(n) << int(shift)


def _at_most_in_a_piece(N, H, dtype, grad):
    """Columns of a piece (forward, backward): statistics or terms of W, dl or terms of W; 2^20 at most."""
    terms = (H + 7) // 8 * 8 * 6 if dtype == "f32" else 0
    dl = N * 2 * (1 if grad == "bf16" else 3)                          # (bf16 gradients of many positions: so much per term)
    return tuple(min(1 << 20, _piece_bytes() // max(x, terms)) for x in (N * 16 // 64, dl))


@pytest.mark.parametrize("N, H, V, dtype, grad, K, pieces", [
    (140, 512, 180001, "f32", "f32", 0, (3, 3)), (140, 512, 180001, "f32", "f32", 7, (3, 3)),            # terms of W, both passes
    (9000, 64, 130003, "bf16", "f32", 0, (2, 2)), (9000, 64, 260003, "bf16", "bf16", 4, (3, 3)),           # statistics and dl
    (40, 8, (1 << 20) + 5, "bf16", "f32", 0, (2, 2)), (140, 8, (2 << 20) + 300, "f32", "f32", 0, (3, 3))])
def test_pieces_of_the_vocabulary(N, H, V, dtype, grad, K, pieces):
    assert all(V > (p - 1) * most for p, most in zip(pieces, _at_most_in_a_piece(N, H, dtype, grad)))
    c = Case(N, H, V, dtype, grad, K=K, tau=2.0, seed=3, g=1.0, spread=2.0)
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    o = _in_64_bits(c, c.h_d, c.y_d)
    # norms: fp32 sums of up to 10^6 terms of either sign, 2^-24 sqrt(10^6); bf16 gradients: their rounding
    for k in ("tok_loss", "dh", "dW", "db") + (("tok_distill",) if K else ()):
        off = float((c.out[k].double() - o[k]).norm() / o[k].norm())
        assert off < (17 / 16 * BF if grad == "bf16" and k in ("dh", "dW", "db") else 1000 * U), (k, off)
        if k in ("dW", "db"):                                          # each piece by itself: none is lost among the others
            for at in torch.arange(V, device="cuda").split(1 << 16):
                part = o[k][at].norm()
                assert float((c.out[k][at].double() - o[k][at]).norm() / part) < (17 / 16 * BF if grad == "bf16" else 2000 * U), (k, int(at[0]))
    for k in ("loss_sum", "distill_sum")[:2 if K else 1]:
        want = float(o["tok_loss" if k == "loss_sum" else "tok_distill"].sum())
        assert abs(float(c.out[k]) - want) < 1e-5 * abs(want)
    if not K:
        word = torch.from_numpy(c.word).cuda()
        W, b, got = c.W.cuda().double(), c.b.cuda().double(), c.out["argmax"].long()
        assert (got[~word] == c.pad_id).all()
        reach = set()
        for at in torch.nonzero(word)[:, 0].split(500):
            l = c.h_d[at].double() @ W.t() + b
            # (logits off by 2^-24 (6 H + 8) times their terms' magnitudes, twice)
            El = 2 * (6 * H + 8) * U * (c.h_d[at].double().abs() @ W.abs().t() + b.abs()).max(1).values
            assert (l.gather(1, got[at][:, None])[:, 0] + 2 * El >= l.max(1).values).all()
            reach |= set((got[at] * pieces[0] // V).tolist())
        assert len(reach) == pieces[0]                                 # maxima lie in every piece
    _untouched(*c.bases.values())


# Equal words next to each other, in one strip of 64 columns and in tiles far apart, in the 64 x 64, 128 x 128 and 256 x 256 kernels and those for few rows
@pytest.mark.parametrize("N, H, V, dtype", [(20, 40, 1000, "f32"), (30, 64, 1000, "bf16"), (40, 64, 400, "bf16"), (700, 72, 8004, "bf16"), (300, 40, 6000, "f32"),
                                            (2100, 64, 33000, "bf16"), (2100, 40, 33000, "f32")])
def test_the_lowest_of_equal_words_wins_in_all_kernels(N, H, V, dtype):
    c = Case(N, H, V, dtype, "f32", pad=0.1, seed=N)
    same = (np.arange(V) % (V // 2)) // 2 * 2                           # words v, v + 1 and both V / 2 further on, v even
    c.W, c.b = c.W[same], c.b[same]
    c.W64, c.b64 = c.W.double().numpy(), c.b.double().numpy()
    v = c.device()
    c.fwd(v)
    got = c.out["argmax"][torch.from_numpy(c.word).cuda()]
    assert (got < V // 2).all() and (got % 2 == 0).all()
    c.check(back=False)


# The lowest temperature: probabilities of nearly 0 and 1
@pytest.mark.parametrize("N, H, V, dtype, grad", [(20, 40, 300, "f32", "f32"), (40, 64, 500, "bf16", "f32"), (700, 72, 4001, "bf16", "bf16")])
def test_the_lowest_temperature(N, H, V, dtype, grad):
    c = Case(N, H, V, dtype, grad, K=6, tau=2.0 ** -10, seed=N)
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    c.check()
    assert all(c.out[k].isfinite().all() for k in ("tok_distill", "dh", "dW", "db"))


# dW and dh in launches of their own, with three words and with none among the positions
@pytest.mark.parametrize("N, H, V, K", [(5000, 1000, 16003, 0), (5000, 1000, 16003, 5), (16384, 2048, 8003, 0)])
def test_a_few_words_or_none_among_many_positions(N, H, V, K):
    y = np.full(N, -1)
    y[[0, N // 2, N - 1]] = [1, V - 1, V // 3]
    c = Case(N, H, V, "bf16", "bf16", K=K, tau=2.0, targets=y, seed=N)
    v = c.device()
    c.fwd(v)
    c.bwd(v)
    o = _in_64_bits(c, c.h_d, c.y_d)
    for k in ("dh", "dW", "db"):
        assert float((c.out[k].double() - o[k]).norm() / o[k].norm()) < 17 / 16 * BF, k
    assert int(c.out["n_tok"]) == 3 and not c.out["dh"][1:N // 2].any()
    c.y_d.fill_(V)
    c.fwd(v)
    c.bwd(v)
    assert int(c.out["n_tok"]) == 0
    for k in ("loss_sum", "tok_loss", "dh", "dW", "db") + (("distill_sum", "tok_distill") if K else ()):
        assert not c.out[k].any(), k
    _untouched(*c.bases.values())
