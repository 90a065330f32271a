"""The attention block over node states, as cases that can be timed and compared.

Three operators and their gradients, each a call of its own:

  norm         layer norm of rows of node states, with the rows' mean and reciprocal deviation
  norm_grad    its gradient: the states' (the residual branch's added), the weights' and the bias's sums over the rows
  linear       act(x W^T + b) + r, the value before the activation kept for the gradient where one will follow
  linear_grad  its gradient: through the activation, then the input's, the weights' and the bias's
  attend       cross attention: the rows of query sequences against the rows of key sequences of other lengths, found by
               lists of pool rows, heads in groups, keys masked, key sequences shared
  attend_grad  its gradient for queries, keys and values

`prepare` makes the inputs from the seed; `run` is one pass, in its plain form or (`own`) as calls of the library;
`exact` is the same pass in 64 bits, written from the definitions.
"""
import math

import torch

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _named(name, c):
    return dict(c, name=name) if name else c


def _norm(name, rows, width, dtype):
    return _named(name, dict(op="norm", rows=rows, width=width, dtype=dtype))


def _norm_grad(name, rows, width, dtype, upstream, residual):
    return _named(name, dict(op="norm_grad", rows=rows, width=width, dtype=dtype, upstream=upstream,
                             residual=residual))


def _linear(name, rows, n_in, n_out, dtype, act, residual, keep):
    return _named(name, dict(op="linear", rows=rows, n_in=n_in, n_out=n_out, dtype=dtype, act=act, residual=residual,
                             keep=keep))


def _linear_grad(name, rows, n_in, n_out, dtype, act):
    return _named(name, dict(op="linear_grad", rows=rows, n_in=n_in, n_out=n_out, dtype=dtype, act=act))


def _attend(name, grad, seqs, share, q_lo, q_hi, k_lo, k_hi, heads, kv_heads, head_dim, dtype, mask, packed):
    return _named(name, dict(op="attend_grad" if grad else "attend", seqs=seqs, share=share, q_lo=q_lo, q_hi=q_hi,
                             k_lo=k_lo, k_hi=k_hi, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
                             mask=mask, packed=packed))


def listed():
    return [
        # The roots of a small served batch, of an odd width: one launch, where latency counts.
        _norm("norm_roots_h300_bf16", 33, 300, "bf16"),
        # The pool of a large batch of trees.
        _norm("norm_pool_h1024_bf16", 131072, 1024, "bf16"),
        # An fp32 model's pool in training, without a residual branch.
        _norm_grad("norm_grad_pool_h512_f32", 55911, 512, "f32", "f32", False),
        # The large bf16 batch: gradients arrive in bf16 and the residual branch's is added on the way.
        _norm_grad("norm_grad_pool_h1024_bf16", 65536, 1024, "bf16", "bf16", True),
        # One state served through the wide layer of a block: reading W is everything.
        _linear("linear_one_h1024_bf16", 1, 1024, 4096, "bf16", "gelu", False, False),
        # Every step of a batch of chains through the block's second layer, added to the branch that goes by it.
        _linear("linear_chains_h1024_bf16", 16384, 4096, 1024, "bf16", "none", True, False),
        # An fp32 model of odd sizes in training.
        _linear_grad("linear_grad_h300_f32", 2049, 300, 1200, "f32", "tanh"),
        # The large batch's wide layer in training.
        _linear_grad("linear_grad_chains_h1024_bf16", 16384, 1024, 4096, "bf16", "gelu"),
        # Serving: one new state of each of 64 chains against documents of up to 4,096 nodes, four heads to one of keys.
        _attend("attend_one_h1024_bf16", False, 64, 1, 1, 1, 512, 4096, 16, 4, 64, "bf16", False, True),
        # Chains against trees in training, padded and pruned nodes masked.
        _attend("attend_trees_h1024_bf16", False, 256, 1, 16, 256, 64, 512, 8, 8, 128, "bf16", True, False),
        # A small fp32 model of an odd head width, four answers for each tree.
        _attend("attend_grad_trees_h300_f32", True, 64, 4, 1, 60, 3, 127, 5, 5, 60, "f32", True, False),
        # The large batch: chains against long chains.
        _attend("attend_grad_chains_h1024_bf16", True, 64, 1, 256, 512, 256, 1024, 16, 16, 64, "bf16", False, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "linear", "linear_grad", "attend", "attend_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_grad"):
        rows, width = _log_int(rng, 1, 131072), _width(rng, 16, 4096)
        while rows > 1 and rows * width * (2 if dtype == "f32" else 1) > 1.3e8:
            rows = (rows + 1) // 2
        if op == "norm":
            return _norm(None, rows, width, dtype)
        return _norm_grad(None, rows, width, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5)
    if op in ("linear", "linear_grad"):
        rows, n_in, n_out = _log_int(rng, 1, 16384), _width(rng, 16, 4096), _width(rng, 16, 4096)
        while rows > 1 and float(rows) * n_in * n_out > (6.8e10 if dtype == "bf16" else 1.7e10):
            rows = (rows + 1) // 2
        act = rng.choice(["none", "relu", "tanh", "gelu"])
        if op == "linear":
            return _linear(None, rows, n_in, n_out, dtype, act, rng.random() < 0.5, act != "none" and rng.random() < 0.5)
        return _linear_grad(None, rows, n_in, n_out, dtype, act)
    seqs = _log_int(rng, 1, 256)
    share = rng.choice([1, 1, 2, 5])
    q_hi = 1 if op == "attend" and rng.random() < 0.4 else _log_int(rng, 1, 1024)
    k_hi = _log_int(rng, 1, 4096)
    q_lo, k_lo = rng.randint(max(1, q_hi // 4), q_hi), rng.randint(max(1, k_hi // 4), k_hi)
    kv_heads, group = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 1, 2, 4])
    head_dim = rng.choice([16, 32, 50, 60, 64, 64, 75, 96, 128, 128])
    while seqs > 1 and float(seqs) * kv_heads * group * q_hi * k_hi * head_dim > (3.4e10 if dtype == "bf16" else 0.9e10):
        seqs = (seqs + 1) // 2
    return _attend(None, op == "attend_grad", seqs, share, q_lo, q_hi, k_lo, k_hi, kv_heads * group, kv_heads, head_dim,
                   dtype, rng.random() < 0.4, rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------

def _ld(n):
    return (n + 63) // 64 * 64


def _matrix(g, rows, width, dtype, scale=1.0, shift=0.0):
    """[rows, _ld(width)] with zeros in the pad columns, as the framework lays out its matrices."""
    m = torch.zeros((rows, _ld(width)), dtype=dtype, device="cuda")
    m[:, :width] = (torch.randn((rows, width), generator=g, device="cuda") * scale + shift).to(dtype)
    return m


def _vector(g, n, scale, shift=0.0):
    return torch.randn(n, generator=g, device="cuda") * scale + shift


def _lengths(n, lo, hi):
    """Lengths spread over lo..hi; of many sequences a few have none."""
    out = [lo + int((hi - lo + 1) * (((i + 1) * 0.6180339887498949) % 1.0)) for i in range(n)]
    return [0 if n > 32 and i % 32 == 31 else v for i, v in enumerate(out)]


def _sizes(c):
    sources = (c["seqs"] + c["share"] - 1) // c["share"]
    return _lengths(c["seqs"], c["q_lo"], c["q_hi"]), _lengths(sources, c["k_lo"], c["k_hi"])


def _pool_rows(g, n):
    """The pool rows of n listed nodes: a schedule's order, by depth and then by node."""
    depth = torch.randint(0, 24, (n,), generator=g, device="cuda")
    order = torch.sort(depth, stable=True).indices
    rows = torch.empty(n, dtype=torch.int32, device="cuda")
    rows[order] = torch.arange(n, dtype=torch.int32, device="cuda")
    return rows


def _ptr(lengths):
    p = torch.zeros(len(lengths) + 1, dtype=torch.int32)
    p[1:] = torch.tensor(lengths, dtype=torch.int32).cumsum(0)
    return p.cuda()


def _table(ptr, most):
    """[sequences, most]: the list entries of every sequence, and which of them are there."""
    at = torch.arange(most, device="cuda")
    n = (ptr[1:] - ptr[:-1]).long()
    there = at < n[:, None]
    return torch.where(there, ptr[:-1].long()[:, None] + at, torch.zeros_like(at)), there


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, dt = case, TYPE[case["dtype"]]
    st = {"case": c}
    if c["op"] in ("norm", "norm_grad"):
        rows, n = c["rows"], c["width"]
        st["x"] = _matrix(g, rows, n, dt, 1.0, 0.25)
        st["gamma"], st["beta"] = _vector(g, n, 0.2, 1.0), _vector(g, n, 0.2)
        if c["op"] == "norm_grad":
            st["dy"] = _matrix(g, rows, n, TYPE[c["upstream"]])
            st["residual"] = _matrix(g, rows, n, dt) if c["residual"] else None
            x = st["x"][:, :n].float()
            st["mean"] = x.mean(1)
            st["rstd"] = torch.rsqrt((x - st["mean"][:, None]).square().mean(1) + EPS)
    elif c["op"] in ("linear", "linear_grad"):
        rows, n_in, n_out = c["rows"], c["n_in"], c["n_out"]
        st["x"] = _matrix(g, rows, n_in, dt)
        st["W"] = _matrix(g, n_out, n_in, dt, n_in ** -0.5)
        st["b"] = _vector(g, n_out, 0.2)
        if c["op"] == "linear":
            st["r"] = _matrix(g, rows, n_out, dt) if c["residual"] else None
        else:
            st["z"] = _matrix(g, rows, n_out, dt)
            st["dout"] = _matrix(g, rows, n_out, dt)
        if own:
            from paper_1702_02181_amd import fold as F
            st["layer"] = F.Linear(st["W"], st["b"], n_in, c["act"])
    else:
        ql, kl = _sizes(c)
        nq, nk, d = sum(ql), sum(kl), c["head_dim"]
        st["q_ptr"], st["k_ptr"] = _ptr(ql), _ptr(kl)
        st["q_rows"], st["k_rows"] = _pool_rows(g, nq), _pool_rows(g, nk)
        st["source"] = (torch.arange(c["seqs"], device="cuda") // c["share"]).int()
        wq, wk = c["heads"] * d, c["kv_heads"] * d
        st["q"] = _matrix(g, nq, wq, dt)
        if c["packed"]:  # keys and values side by side, as one layer writes them
            kv = _matrix(g, nk, 2 * wk, dt)
            st["k"], st["v"] = kv[:, :wk], kv[:, wk:2 * wk]
        else:
            st["k"], st["v"] = _matrix(g, nk, wk, dt)[:, :wk], _matrix(g, nk, wk, dt)[:, :wk]
        st["mask"] = None
        if c["mask"]:  # one key in ten is taken out, and all of the first sequence's
            st["mask"] = (torch.rand(nk, generator=g, device="cuda") > 0.1).to(torch.uint8)
            if len(kl) > 1:
                st["mask"][:kl[0]] = 0
        st["tables"] = _table(st["q_ptr"], max(max(ql), 1)) + _table(st["k_ptr"], max(max(kl), 1))
        if c["op"] == "attend_grad":
            o, st["lse"] = _attention(c, st)
            st["out"] = torch.zeros((nq, _ld(wq)), dtype=dt, device="cuda")
            st["out"][:, :wq] = o.to(dt)
            st["dout"] = _matrix(g, nq, wq, dt)
        if own:
            from paper_1702_02181_amd import fold as F
            st["cross"] = F.CrossAttention(c["heads"], d, st["q_ptr"], st["k_ptr"], st["q_rows"], st["k_rows"],
                                           num_query_rows=nq, num_key_rows=nk, source=st["source"],
                                           kv_heads=c["kv_heads"], dtype=dt)
    return st


# ---- one pass -------------------------------------------------------------------------------------------------

def run(st):
    c = st["case"]
    return (_own if own else _plain)[c["op"]](c, st)


def _activate(act, z):
    if act == "relu":
        return z.clamp(min=0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _slope(act, z):
    if act == "relu":
        return (z > 0).float()
    if act == "tanh":
        return 1 - torch.tanh(z).square()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _plain_norm(c, st):
    x = st["x"][:, :c["width"]].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = torch.rsqrt(x.square().mean(1) + EPS)
    y = x * rstd[:, None] * st["gamma"] + st["beta"]
    return {"y": y.to(TYPE[c["dtype"]]), "mean": mean, "rstd": rstd}


def _plain_norm_grad(c, st):
    n = c["width"]
    x, dy = st["x"][:, :n].float(), st["dy"][:, :n].float()
    xh = (x - st["mean"][:, None]) * st["rstd"][:, None]
    g = dy * st["gamma"]
    dx = st["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if c["residual"]:
        dx = dx + st["residual"][:, :n].float()
    return {"dx": dx.to(TYPE[c["dtype"]]), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _plain_linear(c, st):
    dt = TYPE[c["dtype"]]
    z = torch.addmm(st["b"], st["x"][:, :c["n_in"]].float(), st["W"][:, :c["n_in"]].float().t())
    out = _activate(c["act"], z)
    if c["residual"]:
        out = out + st["r"][:, :c["n_out"]].float()
    return {"out": out.to(dt), "z": z.to(dt)} if c["keep"] else {"out": out.to(dt)}


def _plain_linear_grad(c, st):
    dt = TYPE[c["dtype"]]
    dz = st["dout"][:, :c["n_out"]].float()
    if c["act"] != "none":
        dz = dz * _slope(c["act"], st["z"][:, :c["n_out"]].float())
    x, w = st["x"][:, :c["n_in"]].float(), st["W"][:, :c["n_in"]].float()
    return {"dx": (dz @ w).to(dt), "dW": (dz.t() @ x).to(dt), "db": dz.sum(0)}


def _heads(c, st):
    """Queries [sequences, key heads, queries x group, head_dim], keys and values [sequences, key heads, keys, head_dim],
    and which keys count [sequences, 1, 1, keys]."""
    qi, _, ki, k_there = st["tables"]
    d, h, group = c["head_dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    src = st["source"].long()
    q = st["q"][:, :c["heads"] * d].float()[st["q_rows"][qi].long()]
    q = q.view(*qi.shape, h, group, d).permute(0, 2, 1, 3, 4).reshape(qi.shape[0], h, -1, d)
    if st["mask"] is not None:
        k_there = k_there & (st["mask"][ki] != 0)
    rows = st["k_rows"][ki].long()
    take = lambda m: m.float()[rows].view(*ki.shape, h, d).permute(0, 2, 1, 3)[src].contiguous()  # noqa: E731
    return q, take(st["k"]), take(st["v"]), k_there[src][:, None, None, :]


def _listed_rows(c, st, t, group):
    """[sequences, key heads, queries x group, n] to rows [query rows, heads x n]."""
    qi, there, _, _ = st["tables"]
    n = t.shape[-1]
    t = t.view(qi.shape[0], c["kv_heads"], qi.shape[1], group, n).permute(0, 2, 1, 3, 4).reshape(*qi.shape, -1)
    out = torch.empty((st["q_rows"].numel(), t.shape[-1]), device="cuda")
    out[st["q_rows"][qi[there]].long()] = t[there]
    return out


def _attention(c, st):
    q, k, v, counts = _heads(c, st)
    s = (torch.matmul(q, k.transpose(2, 3)) * c["head_dim"] ** -0.5).masked_fill(~counts, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(s - top)
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    group = c["heads"] // c["kv_heads"]
    return _listed_rows(c, st, o, group), _listed_rows(c, st, top + torch.log(total), group)


def _plain_attend(c, st):
    o, lse = _attention(c, st)
    return {"out": o.to(TYPE[c["dtype"]]), "lse": lse}


def _plain_attend_grad(c, st):
    dt, d, group = TYPE[c["dtype"]], c["head_dim"], c["heads"] // c["kv_heads"]
    q, k, v, counts = _heads(c, st)
    qi, there, ki, k_there = st["tables"]
    row = st["q_rows"][qi].long()

    def queries(m, n):
        m = torch.where(there[..., None], m[:, :c["heads"] * n].float()[row], torch.zeros((), device="cuda"))
        return m.view(*qi.shape, c["kv_heads"], group, n).permute(0, 2, 1, 3, 4).reshape(qi.shape[0], c["kv_heads"], -1, n)

    do, lse = queries(st["dout"], d), queries(st["lse"], 1)
    scale = d ** -0.5
    p = torch.exp(torch.matmul(q, k.transpose(2, 3)) * scale - lse)
    p = torch.where(counts, p, torch.zeros((), device="cuda"))
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3))
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * scale
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    rows = st["k_rows"][ki[k_there]].long()

    def keys(t):  # the sequences that read the same keys are summed
        t = torch.zeros((ki.shape[0],) + t.shape[1:], device="cuda").index_add_(0, st["source"].long(), t)
        out = torch.empty((st["k_rows"].numel(), c["kv_heads"] * d), device="cuda")
        out[rows] = t.permute(0, 2, 1, 3).reshape(*ki.shape, -1)[k_there]
        return out.to(dt)

    return {"dq": _listed_rows(c, st, dq, group).to(dt), "dk": keys(dk), "dv": keys(dv)}


def _own_norm(c, st):
    from paper_1702_02181_amd import fold as F
    y, mean, rstd = F.layer_norm(st["x"], c["width"], st["gamma"], st["beta"], EPS)
    return {"y": y[:, :c["width"]], "mean": mean, "rstd": rstd}


def _own_norm_grad(c, st):
    from paper_1702_02181_amd import fold as F
    dx, dgamma, dbeta = F.layer_norm_backward(st["x"], c["width"], st["dy"], st["mean"], st["rstd"], st["gamma"],
                                              residual=st["residual"], dtype=TYPE[c["dtype"]])
    return {"dx": dx[:, :c["width"]], "dgamma": dgamma, "dbeta": dbeta}


def _own_linear(c, st):
    n = c["n_out"]
    if c["keep"]:
        out, z = st["layer"].forward(st["x"], residual=st["r"], pre=True)
        return {"out": out[:, :n], "z": z[:, :n]}
    return {"out": st["layer"].forward(st["x"], residual=st["r"])[:, :n]}


def _own_linear_grad(c, st):
    dt = TYPE[c["dtype"]]
    dx, dw, db = st["layer"].backward(st["x"], st["dout"], pre=None if c["act"] == "none" else st["z"], dx_dtype=dt,
                                      dw_dtype=dt)
    return {"dx": dx[:, :c["n_in"]], "dW": dw[:, :c["n_in"]], "db": db}


def _own_attend(c, st):
    out, lse = st["cross"].forward(st["q"], st["k"], st["v"], key_mask=st["mask"])
    return {"out": out[:, :c["heads"] * c["head_dim"]], "lse": lse}


def _own_attend_grad(c, st):
    dq, dk, dv = st["cross"].backward(st["q"], st["k"], st["v"], st["out"], st["lse"], st["dout"], key_mask=st["mask"])
    wk = c["kv_heads"] * c["head_dim"]
    return {"dq": dq[:, :c["heads"] * c["head_dim"]], "dk": dk[:, :wk], "dv": dv[:, :wk]}


_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "linear": _plain_linear,
          "linear_grad": _plain_linear_grad, "attend": _plain_attend, "attend_grad": _plain_attend_grad}
_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "linear": _own_linear, "linear_grad": _own_linear_grad,
        "attend": _own_attend, "attend_grad": _own_attend_grad}


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(c):
    e = {"f32": 4, "bf16": 2}
    b = e[c["dtype"]]
    if c["op"] in ("norm", "norm_grad"):
        rows, n = c["rows"], c["width"]
        if c["op"] == "norm":
            return {"bytes": 2 * b * rows * n + 8 * rows + 8 * n, "flops": 8.0 * rows * n}
        return {"bytes": (2 * b + e[c["upstream"]] + (b if c["residual"] else 0)) * rows * n + 8 * rows + 12 * n,
                "flops": 14.0 * rows * n}
    if c["op"] in ("linear", "linear_grad"):
        rows, n, m = c["rows"], c["n_in"], c["n_out"]
        if c["op"] == "linear":
            return {"bytes": b * (rows * n + n * m + rows * m * (1 + c["residual"] + c["keep"])) + 4 * m,
                    "flops": 2.0 * rows * n * m}
        return {"bytes": b * (2 * rows * n + 2 * n * m + rows * m * (1 if c["act"] == "none" else 2)) + 4 * m,
                "flops": 4.0 * rows * n * m}
    ql, kl = _sizes(c)
    nq, nk, d, h = sum(ql), sum(kl), c["head_dim"], c["heads"]
    pairs = sum(n * kl[i // c["share"]] for i, n in enumerate(ql))
    rows_q, rows_k = b * nq * h * d, b * nk * c["kv_heads"] * d
    lists = 4 * (nq + nk + 2 * c["seqs"]) + (nk if c["mask"] else 0) + 4 * nq * h
    if c["op"] == "attend":
        return {"bytes": 2 * rows_q + 2 * rows_k + lists, "flops": 4.0 * pairs * h * d}
    return {"bytes": 4 * rows_q + 4 * rows_k + lists, "flops": 10.0 * pairs * h * d}


# ---- in 64 bits, from the definitions -------------------------------------------------------------------------

def exact(c, seed):
    st = prepare(c, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm, "linear": _exact_linear, "linear_grad": _exact_linear,
            "attend": _exact_attend, "attend_grad": _exact_attend}[c["op"]](c, st)


def _exact_norm(c, st):
    """The definition's values, and gradients by automatic differentiation of them, a slice of rows at a time."""
    n, parts, sums = c["width"], [], 0.0
    gamma, beta = st["gamma"].double(), st["beta"].double()
    step = max(1, (1 << 25) // n)
    for lo in range(0, c["rows"], step):
        x = st["x"][lo:lo + step, :n].double()
        if c["op"] == "norm":
            var, mean = torch.var_mean(x, 1, correction=0)
            y = torch.nn.functional.layer_norm(x, (n,), gamma, beta, EPS)
            parts.append((y, mean, (var + EPS) ** -0.5))
            continue
        x.requires_grad_()
        w = [gamma.clone().requires_grad_(), beta.clone().requires_grad_()]
        y = torch.nn.functional.layer_norm(x, (n,), *w, EPS)
        dx, dg, db = torch.autograd.grad(y, [x] + w, st["dy"][lo:lo + step, :n].double())
        parts.append((dx + st["residual"][lo:lo + step, :n].double() if c["residual"] else dx,))
        sums = torch.stack([dg, db]) + sums
    joined = [torch.cat(p) for p in zip(*parts)]
    if c["op"] == "norm":
        return dict(zip(("y", "mean", "rstd"), joined))
    return {"dx": joined[0], "dgamma": sums[0], "dbeta": sums[1]}


def _exact_linear(c, st):
    n, m = c["n_in"], c["n_out"]
    w, b = st["W"][:, :n].double(), st["b"].double()
    act = {"none": lambda z: z, "relu": torch.relu, "tanh": torch.tanh, "gelu": torch.nn.functional.gelu}[c["act"]]
    outs, dw, db = [], 0.0, 0.0
    for lo in range(0, c["rows"], 2048):
        x = st["x"][lo:lo + 2048, :n].double()
        if c["op"] == "linear":
            z = x @ w.t() + b
            y = act(z)
            outs.append((y + st["r"][lo:lo + 2048, :m].double() if c["residual"] else y, z))
            continue
        z = st["z"][lo:lo + 2048, :m].double().requires_grad_()
        (dz,) = torch.autograd.grad(act(z), z, st["dout"][lo:lo + 2048, :m].double())
        outs.append((dz @ w,))
        dw, db = dw + dz.t() @ x, db + dz.sum(0)
    joined = [torch.cat(p) for p in zip(*outs)]
    if c["op"] == "linear":
        return dict(zip(("out", "z"), joined)) if c["keep"] else {"out": joined[0]}
    return {"dx": joined[0], "dW": dw, "db": db}


def _exact_attend(c, st):
    """One sequence after the other, over the keys that count; gradients by automatic differentiation."""
    d, h, group = c["head_dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    grad = c["op"] == "attend_grad"
    q_ptr, k_ptr, src = st["q_ptr"].tolist(), st["k_ptr"].tolist(), st["source"].tolist()
    q, k, v = (st[x].double() for x in ("q", "k", "v"))
    out = torch.zeros((q.shape[0], h * group * d), dtype=torch.float64, device="cuda")
    lse = torch.full((q.shape[0], h * group), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(out), torch.zeros_like(k), torch.zeros_like(v)
    for i, e in enumerate(src):
        rows, keys = st["q_rows"][q_ptr[i]:q_ptr[i + 1]].long(), st["k_rows"][k_ptr[e]:k_ptr[e + 1]].long()
        if st["mask"] is not None:
            keys = keys[st["mask"][k_ptr[e]:k_ptr[e + 1]] != 0]
        if rows.numel() == 0 or keys.numel() == 0:
            continue
        qs = q[rows, :h * group * d].view(-1, h, group, d).permute(1, 2, 0, 3).contiguous()
        ks, vs = (m[keys].view(-1, h, d).permute(1, 0, 2).contiguous() for m in (k, v))
        leaves = [t.requires_grad_(grad) for t in (qs, ks, vs)]
        s = (qs.reshape(h, -1, d) @ ks.transpose(1, 2)).view(h, group, rows.numel(), -1) * d ** -0.5
        o = (torch.softmax(s, 3).reshape(h, -1, keys.numel()) @ vs).view(h, group, -1, d)
        if not grad:
            out[rows] = o.permute(2, 0, 1, 3).reshape(rows.numel(), -1)
            lse[rows] = torch.logsumexp(s, 3).permute(2, 0, 1).reshape(rows.numel(), -1)
            continue
        do = st["dout"][rows, :h * group * d].double().view(-1, h, group, d).permute(1, 2, 0, 3)
        a, b, e_v = torch.autograd.grad(o, leaves, do)
        dq[rows] = a.permute(2, 0, 1, 3).reshape(rows.numel(), -1)
        dk[keys] += b.permute(1, 0, 2).reshape(keys.numel(), -1)
        dv[keys] += e_v.permute(1, 0, 2).reshape(keys.numel(), -1)
    return {"dq": dq, "dk": dk, "dv": dv} if grad else {"out": out, "lse": lse}
