"""The vocabulary head over node states, as cases that can be timed and compared.

Four operators, each a call of its own:

  logits     z = s W^T + b for rows of node states (a pool, or the roots), one output per token of a vocabulary
  backward   from dz: the states' gradient dz W, the weights' dz^T s and the bias's column sums
  distill    the distillation loss against a teacher's top logits, mixed with the cross entropy of a label, and its
             gradient for every logit
  logprobs   log probabilities of given tokens, the entropy of every row and its top alternatives

`prepare` makes the inputs from the seed; `run` is one pass, in its plain form or (`own`) as calls of the library;
`exact` is the same pass in 64 bits, written from the definitions.
"""
import math

import torch

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _logits(name, rows, hidden, vocab, dtype, out):
    c = dict(op="logits", rows=rows, hidden=hidden, vocab=vocab, dtype=dtype, out=out)
    return dict(c, name=name) if name else c


def _backward(name, rows, hidden, vocab, dtype, add):
    c = dict(op="backward", rows=rows, hidden=hidden, vocab=vocab, dtype=dtype, add=add)
    return dict(c, name=name) if name else c


def _distill(name, rows, vocab, dtype, grad, k, temperature, soft, hard):
    c = dict(op="distill", rows=rows, vocab=vocab, dtype=dtype, grad=grad, k=k, temperature=temperature, soft=soft,
             hard=hard)
    return dict(c, name=name) if name else c


def _logprobs(name, rows, vocab, dtype, tokens, top):
    c = dict(op="logprobs", rows=rows, vocab=vocab, dtype=dtype, tokens=tokens, top=top)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One state scored against the vocabulary: a served chain's next token, where reading W is everything.
        _logits("logits_one_h1024_bf16", 1, 1024, 50000, "bf16", "f32"),
        # The roots of a small batch through a head of odd sizes.
        _logits("logits_roots_h300_f32", 257, 300, 20001, "f32", "f32"),
        # Every step of a batch of chains: the large product of training and of scoring whole sequences.
        _logits("logits_chains_h1024_bf16", 8192, 1024, 32000, "bf16", "bf16"),
        # The gradients of a small batch: few rows, so that W and dW are most of the traffic.
        _backward("backward_b33_h300_bf16", 33, 300, 20000, "bf16", False),
        # An fp32 model with weights tied to the leaf table: gradients added to what the table already has.
        _backward("backward_tied_h256_f32", 2048, 256, 10000, "f32", True),
        # The gradients of the large batch.
        _backward("backward_chains_h1024_bf16", 8192, 1024, 32000, "bf16", False),
        # Distillation on a handful of roots, labels mixed in: a small batch, where the launches count.
        _distill("distill_roots_f32", 48, 10000, "f32", "f32", 8, 2.0, 0.7, 0.3),
        # The large batch's loss: bf16 logits in, bf16 gradients out, teacher's top 32 at temperature 2 and labels.
        _distill("distill_chains_bf16", 8192, 32000, "bf16", "bf16", 32, 2.0, 0.5, 0.5),
        # A long vocabulary of an odd size from fp32 logits, soft targets alone.
        _distill("distill_long_f32_bf16", 2048, 130001, "f32", "bf16", 64, 1.0, 1.0, 0.0),
        # A served token: its log probability and five alternatives.
        _logprobs("logprobs_one_f32", 1, 50000, "f32", 1, 5),
        # A serving batch with a long vocabulary, as many alternatives as servers offer.
        _logprobs("logprobs_serve_bf16", 64, 131072, "bf16", 1, 20),
        # Whole sequences scored (perplexity, preference data): the largest read.
        _logprobs("logprobs_score_bf16", 16384, 50000, "bf16", 2, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logits", "backward", "distill", "logprobs"])
    dtype = rng.choice(["f32", "bf16"])
    rows = _log_int(rng, 1, 16384)
    vocab = _log_int(rng, 2 if op in ("distill", "logprobs") else 33, 131072)
    if rng.random() < 0.4:  # vocabularies are often whole multiples of 64
        vocab = max(64, vocab // 64 * 64)
    if op in ("logits", "backward"):
        hidden = _log_int(rng, 16, 1024)
        if rng.random() < 0.6:
            hidden = max(64, hidden // 64 * 64)
        most = 2.6e11 if dtype == "bf16" else 0.4e11  # no more than the listed cases cost
        while rows > 1 and float(rows) * hidden * vocab > most:
            rows = (rows + 1) // 2
        if op == "logits":
            return _logits(None, rows, hidden, vocab, dtype, "f32" if dtype == "f32" else rng.choice(["bf16", "f32"]))
        return _backward(None, rows, hidden, vocab, dtype, rng.random() < 0.5)
    most = 2.6e8 if op == "distill" else 8.0e8
    while rows > 1 and float(rows) * vocab * (2 if dtype == "f32" else 1) > most:
        rows = (rows + 1) // 2
    if op == "distill":
        soft, hard = rng.choice([(1.0, 0.0), (0.5, 0.5), (0.9, 0.1), (0.0, 1.0)])
        return _distill(None, rows, vocab, dtype, "bf16" if dtype == "bf16" else rng.choice(["f32", "bf16"]),
                        _log_int(rng, 1, 128), rng.choice([1.0, 2.0, 4.0]), soft, hard)
    return _logprobs(None, rows, vocab, dtype, rng.randint(1, 4), rng.randint(0, 32))


# ---- inputs ---------------------------------------------------------------------------------------------------

def _ld(width):
    """The row stride of every matrix: the width rounded up to 64, the columns beyond it zero."""
    return (width + 63) // 64 * 64


def _padded(x, dtype):
    out = torch.zeros((x.shape[0], _ld(x.shape[1])), dtype=TYPE[dtype], device="cuda")
    out[:, :x.shape[1]] = x
    return out


def _targets(rows, vocab, g):
    """Tokens of a row: an index into the part of the vocabulary that no mask below covers; -1 in one row of 16."""
    t = torch.randint(0, max(1, 3 * vocab // 4), (rows,), generator=g, device="cuda", dtype=torch.int32)
    return torch.where(torch.rand(rows, generator=g, device="cuda") < 1 / 16, torch.full_like(t, -1), t)


def _masked_logits(c, g):
    """Logits of a trained model's spread; one row in 8 with a quarter of the vocabulary masked away by -inf, one in 8
    by the type's lowest value."""
    rows, vocab = c["rows"], c["vocab"]
    z = _padded(torch.randn((rows, vocab), generator=g, device="cuda").mul_(2.5), c["dtype"])
    at = torch.arange(rows, device="cuda")
    cols = torch.arange(z.shape[1], device="cuda")
    cut = ((cols >= max(1, 3 * vocab // 4)) & (cols < vocab))[None, :]
    for which, value in ((3, -math.inf), (5, torch.finfo(z.dtype).min)):
        z = z.masked_fill((at % 8 == which)[:, None] & cut, value)
    return z


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    st = {"case": c}
    if c["op"] in ("logits", "backward"):
        rows, hidden, vocab, dtype = c["rows"], c["hidden"], c["vocab"], c["dtype"]
        st["states"] = _padded(torch.tanh(rand(rows, hidden)), dtype)
        st["W"] = _padded(rand(vocab, hidden).mul_(3.0 / math.sqrt(hidden)), dtype)
        st["bias"] = rand(vocab).mul_(0.5)
    if c["op"] == "backward":
        p = torch.softmax(rand(rows, vocab).mul_(2.0), 1)
        y = _targets(rows, vocab, g).long()
        p.scatter_add_(1, y.clamp(min=0)[:, None], torch.full((rows, 1), -1.0, device="cuda"))
        p *= ((y >= 0) / rows)[:, None]  # the mean's gradient; rows without a label have none
        st["dz"] = _padded(p, dtype)
        if c["add"]:
            st["dW"] = _padded(rand(vocab, hidden).mul_(1e-3), "f32")
            st["db"] = rand(vocab).mul_(1e-3)
    if c["op"] == "distill":
        rows, vocab, k = c["rows"], c["vocab"], c["k"]
        st["z"] = _masked_logits(c, g)
        tok = torch.randint(0, max(1, 3 * vocab // 4), (rows, k), generator=g, device="cuda", dtype=torch.int32)
        t = rand(rows, k).mul_(3.0).sort(dim=1, descending=True).values
        have = torch.randint(0, k + 1, (rows,), generator=g, device="cuda")  # a teacher may give fewer than k
        have = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.8, torch.full_like(have, k), have)
        tok = torch.where(torch.arange(k, device="cuda")[None, :] < have[:, None], tok, torch.full_like(tok, -1))
        st["tok"], st["t"] = tok.contiguous(), t.contiguous()
        st["y"] = _targets(rows, vocab, g) if c["hard"] else None
        st["scale"] = 1.0 / rows
    if c["op"] == "logprobs":
        st["z"] = _masked_logits(c, g)
        if c["rows"] > 8:
            st["z"][7::64, :c["vocab"]] = -math.inf  # rows whose mask leaves nothing
        st["tok"] = torch.stack([_targets(c["rows"], c["vocab"], g) for _ in range(c["tokens"])], 1).contiguous()
    return st


# ---- one pass -------------------------------------------------------------------------------------------------

def run(st):
    c = st["case"]
    return (_own if own else _plain)[c["op"]](c, st)


def _plain_logits(c, st):
    z = st["states"].float() @ st["W"].float().t() + st["bias"]
    return {"z": z.to(TYPE[c["out"]])}


def _plain_backward(c, st):
    s, w, dz = st["states"][:, :c["hidden"]].float(), st["W"][:, :c["hidden"]].float(), st["dz"][:, :c["vocab"]].float()
    ds, dw, db = dz @ w, dz.t() @ s, dz.sum(0)
    if c["add"]:
        dw, db = st["dW"][:, :c["hidden"]] + dw, st["db"] + db
    return {"ds": ds, "dW": dw, "db": db}


def _plain_distill(c, st):
    z, T = st["z"][:, :c["vocab"]].float(), c["temperature"]
    tok = st["tok"].long()
    have = tok >= 0
    at = tok.clamp(min=0)
    t = torch.where(have, st["t"] / T, torch.full_like(st["t"], -math.inf))
    some = have.any(1)
    q = torch.where(some[:, None], torch.softmax(t, 1), torch.zeros_like(t)).nan_to_num(0.0)
    zt = z / T
    logp = zt - torch.logsumexp(zt, 1, keepdim=True)
    kl = torch.where(q > 0, q * (torch.log(q) - logp.gather(1, at)), torch.zeros_like(q)).sum(1)
    loss = c["soft"] * T * T * kl
    d = c["soft"] * T * some[:, None] * torch.exp(logp)
    d.scatter_add_(1, at, -c["soft"] * T * q)
    if c["hard"]:
        y = st["y"].long()
        lab, ya = y >= 0, y.clamp(min=0)[:, None]
        logp1 = z - torch.logsumexp(z, 1, keepdim=True)
        loss = loss + torch.where(lab, -c["hard"] * logp1.gather(1, ya)[:, 0], torch.zeros_like(loss))
        d += c["hard"] * lab[:, None] * torch.exp(logp1)
        d.scatter_add_(1, ya, -c["hard"] * lab[:, None].float())
    return {"loss": loss, "dz": (st["scale"] * d).to(TYPE[c["grad"]])}


def _plain_logprobs(c, st):
    z, vocab = st["z"][:, :c["vocab"]].float(), c["vocab"]
    m = z.amax(1, keepdim=True)
    empty = torch.isinf(m)
    x = z - torch.where(empty, torch.zeros_like(m), m)
    e = torch.exp(x)
    s = torch.where(empty, torch.ones_like(m), e.sum(1, keepdim=True))
    lse = torch.where(empty, torch.zeros_like(m), m + torch.log(s))
    ent = torch.log(s[:, 0]) - torch.where(e > 0, e * x, torch.zeros_like(e)).sum(1) / s[:, 0]
    tok = st["tok"].long()
    lp = torch.where(tok >= 0, z.gather(1, tok.clamp(min=0)) - lse, torch.zeros((), device="cuda"))
    out = {"logp": lp, "entropy": ent}
    if c["top"]:
        # one whole-number key a logit, its order first and then the lowest index
        b = (z + 0.0).view(torch.int32).long()
        key = torch.where(b >= 0, b, -(b & 0x7FFFFFFF)) * (1 << 32) + ((1 << 31) - 1 - torch.arange(vocab, device="cuda"))
        k = min(c["top"], vocab)
        at = (1 << 31) - 1 - (key.topk(k, 1).values & 0xFFFFFFFF)
        v = z.gather(1, at)
        at = torch.where(torch.isinf(v), torch.full_like(at, -1), at)
        v = v - lse
        pad = (0, c["top"] - k)
        out["top"] = torch.nn.functional.pad(at, pad, value=-1).int()
        out["top_logp"] = torch.nn.functional.pad(v, pad, value=-math.inf)
    return out


def _own_logits(c, st):
    from paper_1702_02181_amd import fold as F
    head = F.VocabHead(st["W"], st["bias"], c["hidden"])
    return {"z": head.logits(st["states"], dtype=TYPE[c["out"]])[:, :c["vocab"]]}


def _own_backward(c, st):
    from paper_1702_02181_amd import fold as F
    head = F.VocabHead(st["W"], st["bias"], c["hidden"])
    if c["add"]:
        ds, dw, db = head.backward(st["states"], st["dz"], dW=st["dW"].clone(), dbias=st["db"].clone(), accumulate=True)
    else:
        ds, dw, db = head.backward(st["states"], st["dz"])
    return {"ds": ds[:, :c["hidden"]], "dW": dw[:, :c["hidden"]], "db": db}


def _own_distill(c, st):
    from paper_1702_02181_amd import fold as F
    loss, dz = F.distill_loss(st["z"], c["vocab"], st["tok"], st["t"], st["y"], temperature=c["temperature"],
                              soft_weight=c["soft"], hard_weight=c["hard"], scale=st["scale"],
                              grad_dtype=TYPE[c["grad"]])
    return {"loss": loss, "dz": dz[:, :c["vocab"]]}


def _own_logprobs(c, st):
    from paper_1702_02181_amd import fold as F
    r = F.token_logprobs(st["z"], c["vocab"], st["tok"], top_k=c["top"])
    out = {"logp": r.logp, "entropy": r.entropy}
    if c["top"]:
        out["top"], out["top_logp"] = r.top_token, r.top_logp
    return out


_plain = {"logits": _plain_logits, "backward": _plain_backward, "distill": _plain_distill, "logprobs": _plain_logprobs}
_own = {"logits": _own_logits, "backward": _own_backward, "distill": _own_distill, "logprobs": _own_logprobs}


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(c):
    size = {"f32": 4, "bf16": 2}
    rows, vocab, e = c["rows"], c["vocab"], size[c["dtype"]]
    if c["op"] == "logits":
        h = c["hidden"]
        return {"bytes": e * h * (rows + vocab) + 4 * vocab + size[c["out"]] * rows * vocab,
                "flops": 2.0 * rows * h * vocab}
    if c["op"] == "backward":
        h = c["hidden"]
        more = 4 * vocab * (h + 1) if c["add"] else 0
        return {"bytes": e * (rows * vocab + h * (rows + vocab)) + 4 * (rows * h + vocab * h + vocab) + more,
                "flops": 4.0 * rows * h * vocab}
    if c["op"] == "distill":
        return {"bytes": (e + size[c["grad"]]) * rows * vocab + rows * (8 * c["k"] + 8), "flops": 8.0 * rows * vocab}
    return {"bytes": e * rows * vocab + rows * (8 * c["tokens"] + 4 + 8 * c["top"]), "flops": 6.0 * rows * vocab}


# ---- in 64 bits, from the definitions -------------------------------------------------------------------------

def exact(c, seed):
    st = prepare(c, seed)
    return {"logits": _exact_logits, "backward": _exact_backward, "distill": _exact_distill,
            "logprobs": _exact_logprobs}[c["op"]](c, st)


def _exact_logits(c, st):
    h = c["hidden"]
    w = st["W"][:, :h].double()
    return {"z": torch.cat([torch.addmm(st["bias"].double(), s[:, :h].double(), w.t())
                            for s in st["states"].split(1024)])}


def _exact_backward(c, st):
    h, v = c["hidden"], c["vocab"]
    w = st["W"][:, :h].double()
    ds, dw, db = [], torch.zeros((v, h), dtype=torch.float64, device="cuda"), 0.0
    if c["add"]:
        dw, db = st["dW"][:, :h].double(), st["db"].double()
    for s, d in zip(st["states"].split(1024), st["dz"].split(1024)):
        d = d[:, :v].double()
        ds.append(d @ w)
        dw = dw + d.t() @ s[:, :h].double()
        db = db + d.sum(0)
    return {"ds": torch.cat(ds), "dW": dw, "db": db}


def _exact_distill(c, st):
    """The loss of the definition, one slice of rows at a time; its gradient by automatic differentiation."""
    T, losses, grads = c["temperature"], [], []
    step = max(1, (1 << 26) // c["vocab"])
    for lo in range(0, c["rows"], step):
        z = st["z"][lo:lo + step, :c["vocab"]].double().requires_grad_()
        tok, t = st["tok"][lo:lo + step].long(), st["t"][lo:lo + step].double()
        here = (tok >= 0).double()
        w = torch.exp((t - t.amax(1, keepdim=True)) / T) * here
        q = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        lp = torch.log_softmax(z / T, 1).gather(1, tok.clamp(min=0))
        row = c["soft"] * T ** 2 * (torch.xlogy(q, q) - q * lp).sum(1)
        if c["hard"]:
            y = st["y"][lo:lo + step].long()
            row = row + c["hard"] * torch.nn.functional.cross_entropy(z, y, ignore_index=-1, reduction="none")
        (d,) = torch.autograd.grad(st["scale"] * row.sum(), z)
        losses.append(row.detach())
        grads.append(d)
    return {"loss": torch.cat(losses), "dz": torch.cat(grads)}


def _exact_logprobs(c, st):
    outs = []
    step = max(1, (1 << 26) // c["vocab"])
    for lo in range(0, c["rows"], step):
        z = st["z"][lo:lo + step, :c["vocab"]].double()
        empty = (z == -math.inf).all(1, keepdim=True)
        lp = torch.log_softmax(torch.where(empty, torch.zeros_like(z), z), 1)
        lp = torch.where(empty, torch.full_like(lp, -math.inf), lp)
        p = torch.exp(lp)
        tok = st["tok"][lo:lo + step].long()
        o = {"logp": torch.where(tok >= 0, lp.gather(1, tok.clamp(min=0)), torch.zeros((), dtype=torch.float64, device="cuda")),
             "entropy": -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)}
        if c["top"]:
            k = min(c["top"], c["vocab"])
            o["top_logp"] = torch.nn.functional.pad(lp.topk(k, 1).values, (0, c["top"] - k), value=-math.inf)
        outs.append(o)
    done = {k: torch.cat([o[k] for o in outs]) for k in outs[0]}
    return {**done, "top": None} if c["top"] else done
