"""What the equations fix about the oracle of the operators over the vocabulary, and what the library refuses before any
launch (no GPU)."""
import os
import re

import numpy as np
import pytest

import paper_1909_00562_amd as lib
from oracle import vocab_ops_oracle as oracle
from paper_1909_00562_amd import binding as bd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _case(seed, N=7, H=5, V=11, K=4):
    r = np.random.default_rng(seed)
    h, W, b = r.normal(size=(N, H)), r.normal(size=(V, H)), r.normal(size=V)
    y = r.integers(1, V, size=N)
    y[2], y[4] = 0, -3
    ids = r.integers(0, V, size=(N, K))
    ids[1] = -1
    ids[3, 1] = ids[3, 0]
    z = r.normal(size=(N, K)) * 2
    z[0, 2] = -np.inf
    return h, W, b, y, (ids, z, 1.7, 0.6)


def _total(h, W, b, y, teacher, g=0.8):
    o = oracle.loss(h, W, b, y, 0, g, teacher)
    return g * o["loss_sum"] + (teacher[3] * o["distill_sum"] if teacher else 0.0)


@pytest.mark.parametrize("with_teacher", [False, True])
def test_gradients_are_those_of_the_losses(with_teacher):
    h, W, b, y, t = _case(3)
    t = t if with_teacher else None
    o = oracle.loss(h, W, b, y, 0, 0.8, t)
    eps = 1e-5
    for name, x in (("dh", h), ("dW", W), ("db", b)):
        for at in np.ndindex(x.shape):
            keep = x[at]
            x[at] = keep + eps
            up = _total(h, W, b, y, t)
            x[at] = keep - eps
            down = _total(h, W, b, y, t)
            x[at] = keep
            assert abs((up - down) / (2 * eps) - o[name][at]) < 1e-8


def test_rows_of_the_derivative_sum_to_zero_and_vanish_at_padding():
    h, W, b, y, t = _case(5)
    h[2], h[4] = np.nan, np.inf
    o = oracle.loss(h, W, b, y, 0, 0.8, t)
    assert np.abs(o["dl"].sum(axis=1)).max() < 1e-14
    for n in (2, 4):
        assert not o["dl"][n].any() and not o["dh"][n].any() and o["tok_loss"][n] == 0 and o["argmax"][n] == 0
    assert np.isfinite(o["dW"]).all() and o["n_tok"] == 5


def test_a_teacher_that_agrees_costs_nothing():
    h, W, b, y, _ = _case(6, K=11)
    ids = np.tile(np.arange(11), (7, 1))
    z = h @ W.T + b
    o = oracle.loss(h, W, b, y, 0, 0.0, (ids, z, 2.0, 1.0))
    assert np.abs(o["tok_distill"]).max() < 1e-13 and np.abs(o["dl"]).max() < 1e-13


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    r = np.random.default_rng(1)
    table, ids, dy = r.normal(size=(6, 3)), np.array([5, 0, -1, 2, 2, 6, 5]), r.normal(size=(7, 3))
    x = oracle.embed_fwd(table, ids, 1.5, 0)
    d = oracle.embed_bwd(ids, dy, 1.5, 6, 0)
    assert abs((x * dy).sum() - (table * d).sum()) < 1e-12
    assert not x[[1, 2, 5]].any() and not d[[0, 1, 3, 4]].any()


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "vocab_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(vocab_\w+)\s*\(", text))
    assert names == set(bd.VOCAB_EXPORTS)
    handle = lib.load_library()
    for n in names:
        assert getattr(handle, n) is not None


# fake, 16-byte aligned, never dereferenced addresses: every check fails before a launch
A = [0x10000 * (i + 1) for i in range(16)]


def _embed(**kw):
    d = dict(N=5, I=16, V=100, pad_id=0, dtype=bd.AS_BF16, grad_dtype=bd.AS_F32, scale=2.0)
    d.update(kw)
    return bd.VoEmbed(*d.values())


def _shape(**kw):
    d = dict(N=5, H=16, V=100, pad_id=0, dtype=bd.AS_BF16, grad_dtype=bd.AS_F32, grad_scale=1.0)
    d.update(kw)
    return bd.VoShape(*d.values())


NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = 1, 2, 3, 4, 5


@pytest.mark.parametrize("kw, code", [
    (dict(N=0), SHAPE), (dict(N=(1 << 24) + 1), SHAPE), (dict(I=0), SHAPE), (dict(V=0), SHAPE), (dict(pad_id=100), SHAPE),
    (dict(pad_id=-2), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(I=12), ALIGN),
    (dict(dtype=5), DTYPE), (dict(dtype=bd.AS_F32, grad_dtype=bd.AS_BF16), DTYPE), (dict(grad_dtype=-1), DTYPE),
    (dict(I=1 << 16, V=1 << 24), SHAPE)])
def test_embedding_refuses_shapes(kw, code):
    s = _embed(**kw)
    assert bd.vocab_embed_workspace_bytes(s) == 0
    assert bd.vocab_embed_fwd(s, A[0], A[1], A[2], check=False) == code
    assert bd.vocab_embed_bwd(s, A[0], A[1], A[2], 0, A[3], 1 << 40, check=False) == code


def test_embedding_refuses_arguments():
    s = _embed()
    n = bd.vocab_embed_workspace_bytes(s)
    assert n > 0
    assert bd.vocab_embed_fwd(None, A[0], A[1], A[2], check=False) == NULL
    for i in range(3):
        a = [A[0], A[1], A[2]]
        a[i] = None
        assert bd.vocab_embed_fwd(s, *a, check=False) == NULL
        a[i] = A[i] + 4
        assert bd.vocab_embed_fwd(s, *a, check=False) == ALIGN
    for i in range(4):
        a = [A[0], A[1], A[2], A[3]]
        a[i] = None
        assert bd.vocab_embed_bwd(s, a[0], a[1], a[2], 0, a[3], n, check=False) == NULL
        a[i] = A[i] + 8
        assert bd.vocab_embed_bwd(s, a[0], a[1], a[2], 0, a[3], n, check=False) == ALIGN
    assert bd.vocab_embed_bwd(s, A[0], A[1], A[2], 0, A[3], n - 1, check=False) == WORKSPACE
    assert bd.vocab_embed_bwd(s, A[0], A[1], A[2], 2, A[3], n, check=False) == SHAPE


@pytest.mark.parametrize("kw, code", [
    (dict(N=0), SHAPE), (dict(N=(1 << 24) + 1), SHAPE), (dict(H=0), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 26) + 1), SHAPE),
    (dict(pad_id=100), SHAPE), (dict(pad_id=-2), SHAPE), (dict(grad_scale=float("nan")), SHAPE), (dict(H=12), ALIGN),
    (dict(dtype=2), DTYPE), (dict(dtype=bd.AS_F32, grad_dtype=bd.AS_BF16), DTYPE), (dict(H=1 << 16, V=1 << 24), SHAPE)])
def test_losses_refuse_shapes(kw, code):
    s, t = _shape(**kw), bd.VoTeacher(4, 1.0, 1.0)
    assert bd.vocab_xent_workspace_bytes(s) == 0 and bd.vocab_xent_workspace_bytes(s, t) == 0
    assert bd.vocab_xent_fwd(s, *A[:8], A[8], 1 << 50, check=False) == code
    assert bd.vocab_xent_bwd(s, A[0], A[1], A[2], 1 << 50, A[3], A[4], A[5], check=False) == code
    assert bd.vocab_distill_fwd(s, t, *A[:12], 1 << 50, check=False) == code
    assert bd.vocab_distill_bwd(s, t, A[0], A[1], A[2], 1 << 50, A[3], A[4], A[5], check=False) == code


@pytest.mark.parametrize("teacher", [(0, 1.0, 1.0), (257, 1.0, 1.0), (4, 0.0, 1.0), (4, -1.0, 1.0), (4, float("nan"), 1.0),
                                     (4, float("inf"), 1.0), (4, 1e-45, 1.0), (4, 1.0, float("nan"))])
def test_losses_refuse_teachers(teacher):
    s, t = _shape(), bd.VoTeacher(*teacher)
    assert bd.vocab_xent_workspace_bytes(s, t) == 0
    assert bd.vocab_distill_fwd(s, t, *A[:12], 1 << 50, check=False) == SHAPE
    assert bd.vocab_distill_bwd(s, t, A[0], A[1], A[2], 1 << 50, A[3], A[4], A[5], check=False) == SHAPE
    assert bd.vocab_xent_workspace_bytes(_shape(V=(1 << 20) + 1), bd.VoTeacher(4, 1.0, 1.0)) == 0


@pytest.mark.parametrize("teacher", [(4, 1e20, 1.0), (4, 1e10, 1e30)])                # tau^2, s tau
def test_losses_refuse_teachers_whose_factors_overflow(teacher):
    s, t = _shape(), bd.VoTeacher(*teacher)
    assert bd.vocab_xent_workspace_bytes(s, t) == 0
    assert bd.vocab_distill_fwd(s, t, *A[:12], 1 << 50, check=False) == SHAPE
    assert bd.vocab_distill_bwd(s, t, A[0], A[1], A[2], 1 << 50, A[3], A[4], A[5], check=False) == SHAPE


def test_losses_refuse_arguments():
    s, t = _shape(), bd.VoTeacher(4, 2.0, 1.0)
    n, nt = bd.vocab_xent_workspace_bytes(s), bd.vocab_xent_workspace_bytes(s, t)
    assert 0 < n < nt
    optional = {2, 6, 7}                            # b, tok_loss, argmax
    for i in range(9):
        a = list(A[:9])
        a[i] += 2
        assert bd.vocab_xent_fwd(s, *a, n, check=False) == ALIGN
        a[i] = None
        if i not in optional:
            assert bd.vocab_xent_fwd(s, *a, n, check=False) == NULL
    assert bd.vocab_xent_fwd(s, *A[:9], n - 1, check=False) == WORKSPACE
    assert "needed" in bd.attn_softmax_last_error()
    optional = {1, 5}                               # b, db
    for i in range(6):
        a = list(A[:6])
        a[i] += 2
        assert bd.vocab_xent_bwd(s, *a[:3], n, *a[3:], check=False) == ALIGN
        a[i] = None
        if i not in optional:
            assert bd.vocab_xent_bwd(s, *a[:3], n, *a[3:], check=False) == NULL
            assert bd.vocab_distill_bwd(s, t, *a[:3], nt, *a[3:], check=False) == NULL
    optional = {2, 9, 10}
    for i in range(12):
        a = list(A[:12])
        a[i] += 2
        assert bd.vocab_distill_fwd(s, t, *a, nt, check=False) == ALIGN
        a[i] = None
        if i not in optional:
            assert bd.vocab_distill_fwd(s, t, *a, nt, check=False) == NULL
    assert bd.vocab_distill_fwd(s, t, *A[:12], nt - 1, check=False) == WORKSPACE
    assert bd.vocab_distill_fwd(s, None, *A[:12], nt, check=False) == NULL
    assert bd.vocab_xent_fwd(None, *A[:9], n, check=False) == NULL


def test_workspace_holds_pieces_of_the_logits_and_not_all_of_them():
    s = _shape(N=16384, H=2048, V=128000, grad_dtype=bd.AS_BF16)
    assert bd.vocab_xent_workspace_bytes(s) < 0.25 * 16384 * 128000 * 2


def test_handles_refuse_tensors_of_the_host_and_types_they_do_not_know():
    torch = pytest.importorskip("torch")
    W = torch.zeros(10, 8)
    with pytest.raises(lib.AttnSoftmaxError, match="AS_ERR_SHAPE"):
        lib.DeviceEmbed(W, 4)
    with pytest.raises(lib.AttnSoftmaxError, match="AS_ERR_SHAPE"):
        lib.DeviceVocabLoss(W, None, 4)
    with pytest.raises(lib.AttnSoftmaxError, match="AS_ERR_DTYPE"):
        bd._grad_dtype("fp32", bd.AS_F32)
