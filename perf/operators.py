"""The operators over the vocabulary as cases that can be timed and compared.

Three operators at the two ends of a model over words, and what each is in its plain form:

  embed    x = scale * table[ids] for the words of a batch (zeros at padding); its gradient adds the rows of dy up per word
  xent     softmax cross-entropy of h W^T + b against word ids without keeping the logits; gradients of h, W and b
  distill  the same with a teacher's top K logits per position as a second, soft target at a temperature

A case with `back` is a training step (forward and all gradients), one without the forward pass alone.  `own` chooses between the
plain form in elementary torch operations and the calls into `paper_1909_00562_amd`.

States are tanh(N(0,1)), weights U(-w, w), words Zipf-like, as in synth_inputs.py; a share `pad` of the positions is padding,
where states may hold anything (here NaN, which no output may show).
"""
import math

import torch

own = False

PAD = 0
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one step of interactive decoding: the words of a few sentences
        dict(name="embed_decode", op="embed", N=16, I=512, V=32000, dtype="bf16", grad="f32", pad=0.0, back=False),
        # the paper's model: embedding 512, 50 steps of 128 right-padded sentences; dx of the LSTM stack is float
        dict(name="embed_mid", op="embed", N=6400, I=512, V=32000, dtype="bf16", grad="f32", pad=0.3, back=True),
        # a small batch whose sizes fit nothing, gradients in the storage type
        dict(name="embed_ragged", op="embed", N=1237, I=1000, V=32003, dtype="bf16", grad="bf16", pad=0.25, back=True),
        # a long packed batch over a large vocabulary, fp32 training
        dict(name="embed_large", op="embed", N=131072, I=1024, V=128000, dtype="f32", grad="f32", pad=0.0, back=True),
        # one decoder step of a small model: the best word and the scores of given ones
        dict(name="xent_decode", op="xent", N=16, H=512, V=32000, dtype="bf16", grad="f32", pad=0.0, back=False),
        # the smallest training of the benchmark in fp32
        dict(name="xent_small_f32", op="xent", N=1920, H=512, V=16000, dtype="f32", grad="f32", pad=0.25, back=True),
        # odd sizes, float gradients of bf16 states (what lstm_stack_bwd and Adam read)
        dict(name="xent_ragged", op="xent", N=2257, H=1000, V=32003, dtype="bf16", grad="f32", pad=0.3, back=True),
        # the paper's model size
        dict(name="xent_mid", op="xent", N=6400, H=1024, V=32000, dtype="bf16", grad="bf16", pad=0.3, back=True),
        # the largest configuration of the benchmark
        dict(name="xent_stress", op="xent", N=16384, H=2048, V=128000, dtype="bf16", grad="bf16", pad=0.25, back=True),
        # a student of the small model in fp32, few teacher logits
        dict(name="distill_small_f32", op="distill", N=640, H=512, V=16000, dtype="f32", grad="f32", pad=0.25, back=True, K=8, tau=1.0),
        # validation of a student: both losses, no gradients
        dict(name="distill_score", op="distill", N=777, H=512, V=32003, dtype="bf16", grad="f32", pad=0.2, back=False, K=20, tau=4.0),
        # a student of the paper's size against a teacher's 64 best words
        dict(name="distill_mid", op="distill", N=6400, H=1024, V=32000, dtype="bf16", grad="bf16", pad=0.3, back=True, K=64, tau=2.0),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "xent", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    grad = "f32" if dtype == "f32" else rng.choice(["f32", "bf16"])
    back = rng.random() < 0.7
    pad = rng.choice([0.0, rng.uniform(0.05, 0.6)])
    if op == "embed":
        I = _log(rng, 64, 2048)
        if dtype == "bf16":
            I = I // 8 * 8
        return dict(op=op, N=_log(rng, 1, 131072 * 1024 // max(I, 1024)), I=I, V=_log(rng, 1000, 128000), dtype=dtype, grad=grad, pad=pad, back=back)
    H = _log(rng, 128, 2048 if dtype == "bf16" else 1024)
    if dtype == "bf16":
        H = H // 8 * 8
    V = _log(rng, 1000, 128000)
    most = 16384 if dtype == "bf16" else 4096
    N = _log(rng, 1, max(1, min(most, int(5e11 if back else 2e12) // (H * V))))
    c = dict(op=op, N=N, H=H, V=V, dtype=dtype, grad=grad, pad=pad, back=back)
    if op == "distill":
        c.update(K=_log(rng, 1, 100), tau=rng.choice([1.0, 2.0, rng.uniform(0.7, 5.0)]))
    return c


def _words(case):
    """How many positions hold a word: one at least."""
    return max(1, case["N"] - int(round(case["N"] * case["pad"])))


def _zipf(shape, V, gen):
    """Words 1..V-1, p(k) about 1/k."""
    u = torch.rand(shape, device=DEV, generator=gen, dtype=torch.float64)
    return torch.exp(u * math.log(V)).to(torch.int32).clamp_(1, V - 1)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    N, V, t, g = case["N"], case["V"], TYPES[case["dtype"]], TYPES[case["grad"]]
    words = _zipf((N,), V, gen)
    # padding: ids that are the pad id or outside the vocabulary
    at_pad = torch.randperm(N, device=DEV, generator=gen)[_words(case):]
    words[at_pad[::2]] = PAD
    words[at_pad[1::2]] = -1
    s = dict(case=case, words=words)
    f32 = dict(device=DEV, dtype=torch.float32)
    uniform = lambda n, m, w: ((torch.rand(n, m, device=DEV, generator=gen) * 2 - 1) * w).to(t)  # noqa: E731
    if case["op"] == "embed":
        I = case["I"]
        s["table"] = uniform(V, I, 0.1)
        s["scale"] = math.sqrt(I)
        s["out"] = torch.empty(N, I, device=DEV, dtype=t)
        if case["back"]:
            s["dy"] = (torch.randn(N, I, device=DEV, generator=gen) * 1e-2).to(g)
            s["dy"][at_pad] = float("nan")
            s["d_table"] = torch.empty(V, I, device=DEV, dtype=g)
        return s
    H = case["H"]
    s["h"] = torch.tanh(torch.randn(N, H, device=DEV, generator=gen)).to(t)
    s["h"][at_pad] = float("nan")
    s["W"] = uniform(V, H, 0.1)
    s["b"] = uniform(1, V, 0.1)[0].contiguous()
    s["loss_sum"], s["n_tok"] = torch.empty(1, **f32), torch.empty(1, device=DEV, dtype=torch.int32)
    s["tok_loss"] = torch.empty(N, **f32)
    s["argmax"] = torch.empty(N, device=DEV, dtype=torch.int32)
    s["g"] = 1.0 / _words(case)
    if case["back"]:
        s["dh"], s["dW"] = torch.empty(N, H, device=DEV, dtype=g), torch.empty(V, H, device=DEV, dtype=g)
        s["db"] = torch.empty(V, device=DEV, dtype=g)
    if case["op"] == "distill":
        K = case["K"]
        s["ids"] = _zipf((N, K), V, gen)
        s["z"] = torch.randn(N, K, device=DEV, generator=gen) * 3 + 5
        # lists shorter than K, and positions that the teacher has not seen: ids outside the vocabulary, logits undefined there
        left = torch.randint(0, K + 1, (N,), device=DEV, generator=gen)
        left = torch.where(torch.rand(N, device=DEV, generator=gen) < 0.8, K, left)
        gone = torch.arange(K, device=DEV)[None, :] >= left[:, None]
        s["ids"][gone] = -1
        s["z"][gone] = float("nan")
        s["distill_sum"], s["tok_distill"] = torch.empty(1, **f32), torch.empty(N, **f32)
        s["distill_scale"] = 0.5 * s["g"]
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------


def _embed_plain(s):
    case, words, table = s["case"], s["words"], s["table"]
    V = table.shape[0]
    word = (words >= 0) & (words < V) & (words != PAD)
    at = torch.where(word, words, 0).long()
    out = torch.where(word[:, None], table[at].float() * s["scale"], 0.0).to(table.dtype)
    if not case["back"]:
        return dict(out=out)
    rows = torch.where(word[:, None], s["dy"].float() * s["scale"], 0.0)
    d = torch.zeros(V, table.shape[1], device=DEV, dtype=torch.float32).index_add_(0, at, rows)
    return dict(out=out, d_table=d.to(s["dy"].dtype))


def _loss_plain(s):
    case, y, soft = s["case"], s["words"], s["case"]["op"] == "distill"
    N, V, gt = case["N"], case["V"], TYPES[case["grad"]]
    word = (y >= 0) & (y < V) & (y != PAD)
    at = torch.where(word, y, 0).long()[:, None]
    h = torch.where(word[:, None], s["h"].float(), 0.0)
    W = s["W"].float()
    l = h @ W.t() + s["b"].float()
    top = l.max(dim=1, keepdim=True)
    lse = top.values + torch.log(torch.exp(l - top.values).sum(dim=1, keepdim=True))
    tok = torch.where(word, (lse - l.gather(1, at))[:, 0], 0.0)
    got = dict(loss_sum=tok.sum(dtype=torch.float64).float()[None], n_tok=word.sum().to(torch.int32)[None], tok_loss=tok)
    if not case["back"] and not soft:
        got["argmax"] = torch.where(word, top.indices[:, 0], PAD).to(torch.int32)
    if soft:
        tau, ids = case["tau"], s["ids"]
        inside = (ids >= 0) & (ids < V) & word[:, None]
        seen = inside.any(dim=1, keepdim=True)
        z = torch.where(inside, s["z"] / tau, -math.inf)
        z = z - torch.where(seen, z.max(dim=1, keepdim=True).values, 0.0)
        e = torch.exp(z)
        total = torch.where(seen, e.sum(dim=1, keepdim=True), 1.0)
        p = e / total
        lse_t = top.values / tau + torch.log(torch.exp((l - top.values) / tau).sum(dim=1, keepdim=True))
        k_at = torch.where(inside, ids, 0).long()
        log_p = torch.where(inside, z - torch.log(total), 0.0)
        log_q = l.gather(1, k_at) / tau - lse_t
        tok_d = tau * tau * (p * (log_p - log_q)).sum(dim=1)
        got.update(distill_sum=tok_d.sum(dtype=torch.float64).float()[None], tok_distill=tok_d)
    if not case["back"]:
        return got
    dl = torch.exp(l - lse)
    dl.scatter_add_(1, at, torch.full_like(lse, -1.0))
    dl *= torch.where(word, s["g"], 0.0)[:, None]
    if soft:
        c = s["distill_scale"] * tau
        l /= tau
        l -= lse_t
        dl += torch.where(seen, c, 0.0) * torch.exp_(l)
        dl.scatter_add_(1, k_at, -c * p)
    got.update(dh=(dl @ W).to(gt), dW=(dl.t() @ h).to(gt), db=dl.sum(dim=0).to(gt))
    return got


# ---- the framework's calls ------------------------------------------------------------------------------------------------


def _embed_own(s):
    import paper_1909_00562_amd as lib
    e = s.get("handle")
    if e is None:   # kept with its workspace, as a program does that trains for more than one step
        e = s["handle"] = lib.DeviceEmbed(s["table"], s["case"]["N"], pad_id=PAD, scale=s["scale"], grad_dtype=s["case"]["grad"])
    e.fwd(s["words"], s["out"])
    if not s["case"]["back"]:
        return dict(out=s["out"])
    e.bwd(s["words"], s["dy"], s["d_table"])
    return dict(out=s["out"], d_table=s["d_table"])


def _loss_own(s):
    import paper_1909_00562_amd as lib
    case, soft = s["case"], s["case"]["op"] == "distill"
    v = s.get("handle")
    if v is None:
        teacher = dict(K=case["K"], temperature=case["tau"], distill_scale=s["distill_scale"]) if soft else {}
        v = s["handle"] = lib.DeviceVocabLoss(s["W"], s["b"], case["N"], pad_id=PAD, grad_scale=s["g"], grad_dtype=case["grad"], **teacher)
    got = dict(loss_sum=s["loss_sum"], n_tok=s["n_tok"], tok_loss=s["tok_loss"])
    if soft:
        v.distill_fwd(s["h"], s["words"], s["ids"], s["z"], s["loss_sum"], s["n_tok"], s["distill_sum"], s["tok_loss"], s["tok_distill"])
        got.update(distill_sum=s["distill_sum"], tok_distill=s["tok_distill"])
    elif case["back"]:
        v.xent_fwd(s["h"], s["words"], s["loss_sum"], s["n_tok"], s["tok_loss"])
    else:
        v.xent_fwd(s["h"], s["words"], s["loss_sum"], s["n_tok"], s["tok_loss"], s["argmax"])
        got["argmax"] = s["argmax"]
    if case["back"]:
        (v.distill_bwd if soft else v.xent_bwd)(s["dh"], s["dW"], s["db"])
        got.update(dh=s["dh"], dW=s["dW"], db=s["db"])
    return got


def run(state):
    if state["case"]["op"] == "embed":
        return _embed_own(state) if own else _embed_plain(state)
    return _loss_own(state) if own else _loss_plain(state)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    N, V = case["N"], case["V"]
    y = s["words"].long()
    rows = torch.nonzero((y > 0) & (y < V))[:, 0]          # (PAD is 0)
    if case["op"] == "embed":
        out = torch.zeros(N, case["I"], device=DEV, dtype=torch.float64)
        out[rows] = s["table"][y[rows]].double() * s["scale"]
        if not case["back"]:
            return dict(out=out)
        d = torch.zeros(V, case["I"], device=DEV, dtype=torch.float64)
        d.index_put_((y[rows],), s["dy"][rows].double() * s["scale"], accumulate=True)
        return dict(out=out, d_table=d)
    soft, tau = case["op"] == "distill", case.get("tau", 1.0)
    W, b = s["W"].double(), s["b"].double()
    zeros = lambda *n: torch.zeros(*n, device=DEV, dtype=torch.float64)  # noqa: E731
    tok, tok_d, dh, dW, db = zeros(N), zeros(N), zeros(N, case["H"]), zeros(V, case["H"]), zeros(V)
    for at in rows.split(1024):
        h = s["h"][at].double()
        l = torch.addmm(b, h, W.t())
        log_q = torch.log_softmax(l, dim=1)
        tok[at] = -log_q[torch.arange(len(at), device=DEV), y[at]]
        dl = torch.softmax(l, dim=1) * s["g"]
        dl[torch.arange(len(at), device=DEV), y[at]] -= s["g"]
        if soft:
            ids = s["ids"][at].long()
            r, k = torch.nonzero((ids >= 0) & (ids < V), as_tuple=True)
            z = torch.full(ids.shape, -math.inf, device=DEV, dtype=torch.float64)
            z[r, k] = s["z"][at].double()[r, k] / tau
            log_p = torch.log_softmax(z, dim=1)[r, k]
            log_qt = torch.log_softmax(l / tau, dim=1)
            tok_d[at] = zeros(len(at)).index_put_((r,), tau * tau * log_p.exp() * (log_p - log_qt[r, ids[r, k]]), accumulate=True)
            known = zeros(len(at)).index_fill_(0, r, 1.0)[:, None]
            p = zeros(len(at), V).index_put_((r, ids[r, k]), log_p.exp(), accumulate=True)
            dl += s["distill_scale"] * tau * (log_qt.exp() * known - p)
        if case["back"]:
            dh[at] = dl @ W
            dW += dl.t() @ h
            db += dl.sum(dim=0)
    got = dict(loss_sum=tok.sum()[None], n_tok=None, tok_loss=tok)
    if soft:
        got.update(distill_sum=tok_d.sum()[None], tok_distill=tok_d)
    if case["back"]:
        got.update(dh=dh, dW=dW, db=db)
    return got


def work(case):
    N, V, R = case["N"], case["V"], _words(case)
    e, g = (4 if case["dtype"] == "f32" else 2), (4 if case["grad"] == "f32" else 2)
    if case["op"] == "embed":
        I = case["I"]
        # (a word's row is read once, however often it comes: about this many different ones of p(k) ~ 1 / k)
        ln = math.log(V)
        different = min(R, V, sum((1 - math.exp(-R * math.log1p(1 / k) / ln)) * w for k, w in _grid(V)))
        moved = 4 * N + different * I * e + N * I * e
        if case["back"]:
            moved += R * I * g + V * I * g
        return dict(bytes=moved, flops=(1 + case["back"]) * R * I)
    H = case["H"]
    moved = R * H * e + V * H * e + V * e + 8 * N
    flops = 2 * R * V * H
    if case["op"] == "distill":
        moved += 8 * R * case["K"] + 4 * N
    if case["back"]:
        moved += N * H * g + V * H * g + V * g
        flops *= 3
    return dict(bytes=moved, flops=flops)


def _grid(V):
    """Words 1..V-1 in groups: (a word of the group, how many it stands for)."""
    k = 1
    while k < V:
        w = max(1, k // 16)
        w = min(w, V - k)
        yield k + (w - 1) / 2, w
        k += w
