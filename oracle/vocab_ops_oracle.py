"""float64 definition of the operators over the vocabulary (include/vocab_ops.h): embedding lookup with scaling, softmax
cross-entropy of a projection, distillation from a teacher's top logits, and their gradients.  One position at a time,
no blocking; shares no code with the library."""
from __future__ import annotations

import numpy as np


def is_word(ids, V, pad_id):
    ids = np.asarray(ids, dtype=np.int64)
    return (ids >= 0) & (ids < V) & (ids != pad_id)


def embed_fwd(table, ids, scale, pad_id):
    table = np.asarray(table, dtype=np.float64)
    out = np.zeros((len(ids), table.shape[1]))
    for n, w in enumerate(ids):
        if is_word(w, table.shape[0], pad_id):
            out[n] = scale * table[w]
    return out


def embed_bwd(ids, dy, scale, V, pad_id, old=None):
    dy = np.asarray(dy, dtype=np.float64)
    d = np.zeros((V, dy.shape[1])) if old is None else np.array(old, dtype=np.float64)
    for n, w in enumerate(ids):
        if is_word(w, V, pad_id):
            d[w] += scale * dy[n]
    return d


def _log_softmax(x):
    m = x.max()
    return x - m - np.log(np.exp(x - m).sum())


def loss(h, W, b, targets, pad_id, grad_scale=1.0, teacher=None):
    """teacher: None or (ids [N,K], logits [N,K], temperature, scale).  Returns a dict of all outputs of the forward and
    the backward pass, and the logits' derivative dl with the logits themselves (l), rows of padding 0."""
    h, W = np.asarray(h, dtype=np.float64), np.asarray(W, dtype=np.float64)
    N, (V, H) = len(targets), W.shape
    b = np.zeros(V) if b is None else np.asarray(b, dtype=np.float64)
    word = is_word(targets, V, pad_id)
    l, dl = np.zeros((N, V)), np.zeros((N, V))
    tok, tok_d = np.zeros(N), np.zeros(N)
    argmax = np.full(N, pad_id, dtype=np.int64)
    for n in np.nonzero(word)[0]:
        l[n] = W @ h[n] + b
        log_q = _log_softmax(l[n])
        tok[n] = -log_q[targets[n]]
        argmax[n] = int(np.argmax(l[n]))          # the lowest of equal ones
        dl[n] = grad_scale * np.exp(log_q)
        dl[n, targets[n]] -= grad_scale
        if teacher is None:
            continue
        ids, z, tau, scale = teacher
        there = [k for k in range(ids.shape[1]) if 0 <= ids[n, k] < V and z[n, k] != -np.inf]
        if not there:
            continue
        log_p = _log_softmax(np.array([float(z[n, k]) for k in there]) / tau)
        log_qt = _log_softmax(l[n] / tau)
        dl[n] += scale * tau * np.exp(log_qt)
        for k, lp in zip(there, log_p):
            p = np.exp(lp)
            if p > 0:
                tok_d[n] += tau * tau * p * (lp - log_qt[ids[n, k]])
            dl[n, ids[n, k]] -= scale * tau * p
    hw = np.where(word[:, None], h, 0.0)           # (rows of padding may hold anything)
    return dict(loss_sum=tok.sum(), n_tok=int(word.sum()), tok_loss=tok, argmax=argmax, distill_sum=tok_d.sum(), tok_distill=tok_d,
                l=l, dl=dl, dh=dl @ W, dW=dl.T @ hw, db=dl.sum(axis=0))
