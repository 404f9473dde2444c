"""Measured cases of the head losses and of the gated norm pair.

Four operators, each in a plain form of elementary torch operations (own = False) and as the
library's own call (own = True):

  xent      softmax cross entropy of hidden states against the vocabulary, with the gradients of the
            hidden states and of the vocabulary matrix, the [T, V] logits not being an output
  distill   the same head learning from a teacher's top logits (k of V) at a temperature
  norm_fwd  norm of a block's output, gated and added to the scaled residual stream, and the norm
            that the next block (or the head) reads
  norm_bwd  its backward pass with every parameter's gradient

With X [T, d], E [V, d], l = X E^T, s = l / temperature and p = softmax(s):

  xent      nll_t = logsumexp(l_t) - l_t[target_t], loss = sum_t w_t nll_t; rows with a negative
            target count nowhere; without weights w_t = 1 / counted rows
  distill   q = softmax over the row's present teacher entries of z / temperature (or, with the
            teacher's own log-sum-exp, exp(z / temperature - lse), which sums to less than one);
            row loss = sum_j q_j (log q_j - log p_j)
  norm      n = N(y) g1 + b1;  r' = a r + gate n;  h = N(r') g2 + b2, N = LayerNorm or RMSNorm

Sizes: the 1.3B- and 125M-class steps and the oracle's tiny model of this repository, and generic
ragged ones around them.
"""
import torch

own = False

EPS = 1e-5
LARGEST_HEAD = 8192 * 2048 * 32768
LARGEST_NORM = 8192 * 2048


def listed():
    return [
        # the head of the 1.3B-class local step: 4 sequences of 2048 tokens, the last position of each without a target
        {"name": "xent_step_1p3b", "op": "xent", "T": 8192, "d": 2048, "V": 32768, "skip": "last", "seq": 2048, "weights": False, "grad": True},
        # a 125M-class batch with masked prompt tokens and weighted rows, odd token count and vocabulary
        {"name": "xent_masked_weighted", "op": "xent", "T": 4099, "d": 768, "V": 32003, "skip": "third", "seq": 1024, "weights": True, "grad": True},
        # evaluation: the loss alone over a large vocabulary
        {"name": "xent_eval_large_vocab", "op": "xent", "T": 2048, "d": 1024, "V": 131075, "skip": "none", "seq": 2048, "weights": False, "grad": False},
        # the tiny model's batch, where launches count
        {"name": "xent_tiny", "op": "xent", "T": 256, "d": 64, "V": 512, "skip": "last", "seq": 64, "weights": False, "grad": True},
        # distilling into the 1.3B-class model from stored top-32 logits
        {"name": "distill_step_1p3b", "op": "distill", "T": 4096, "d": 2048, "V": 32768, "k": 32, "temp": 2.0, "ragged": False, "lse": False, "weights": False, "grad": True},
        # few rows against the whole vocabulary, the teacher's normaliser known
        {"name": "distill_few_rows", "op": "distill", "T": 24, "d": 768, "V": 32768, "k": 64, "temp": 1.0, "ragged": False, "lse": True, "weights": False, "grad": True},
        # odd sizes, rows with fewer entries or none
        {"name": "distill_ragged", "op": "distill", "T": 1001, "d": 520, "V": 5003, "k": 7, "temp": 1.5, "ragged": True, "lse": False, "weights": True, "grad": True},
        # one decoded token
        {"name": "norm_fwd_one_token", "op": "norm_fwd", "T": 1, "d": 2048, "kind": "rms", "shift": False, "gate": "channel", "seq": 1, "scale": 1.0},
        # a layer of the 1.3B-class step
        {"name": "norm_fwd_step_1p3b", "op": "norm_fwd", "T": 8192, "d": 2048, "kind": "layer", "shift": True, "gate": "channel", "seq": 2048, "scale": 0.9},
        {"name": "norm_bwd_step_1p3b", "op": "norm_bwd", "T": 8192, "d": 2048, "kind": "layer", "shift": True, "gate": "channel", "seq": 2048, "scale": 0.9},
        # a gate for each sequence (conditioned blocks), odd lengths
        {"name": "norm_bwd_sequence_gate", "op": "norm_bwd", "T": 13 * 157, "d": 768, "kind": "rms", "shift": False, "gate": "sequence", "seq": 157, "scale": 1.0},
        # a gate for each token
        {"name": "norm_bwd_token_gate", "op": "norm_bwd", "T": 777, "d": 1032, "kind": "layer", "shift": True, "gate": "token", "seq": 1, "scale": 0.5},
    ]


def _log_int(rng, lo, hi):
    import math
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["xent", "distill", "norm_fwd", "norm_bwd"])
    if op in ("xent", "distill"):
        V = _log_int(rng, 300, 131072)
        d = 8 * _log_int(rng, 8, 256)
        T = _log_int(rng, 1, max(1, min(8192, LARGEST_HEAD // (V * d))))
        if op == "xent":
            return {"op": op, "T": T, "d": d, "V": V, "skip": rng.choice(["none", "last", "third"]), "seq": _log_int(rng, 16, 2048),
                    "weights": rng.random() < 0.5, "grad": rng.random() < 0.75}
        return {"op": op, "T": T, "d": d, "V": V, "k": _log_int(rng, 1, 64), "temp": rng.choice([1.0, 1.5, 2.0, 4.0]), "ragged": rng.random() < 0.5,
                "lse": rng.random() < 0.5, "weights": rng.random() < 0.5, "grad": rng.random() < 0.75}
    d = 8 * _log_int(rng, 8, 512)
    T = _log_int(rng, 1, min(16384, LARGEST_NORM // d))
    return {"op": op, "T": T, "d": d, "kind": rng.choice(["layer", "rms"]), "shift": rng.random() < 0.5, "gate": rng.choice(["none", "channel", "sequence", "token"]),
            "seq": _log_int(rng, 2, 2048), "scale": rng.choice([1.0, 0.9, 0.5])}


# ---- inputs -------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gate_rows(case):
    """Rows that share a row of the gate."""
    return {"none": 0, "channel": case["T"], "sequence": case["seq"], "token": 1}[case["gate"]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, d = case["T"], case["d"]
    if case["op"] in ("xent", "distill"):
        V = case["V"]
        # logits with a spread of about 3, the right id raised by about 7: a model that has learnt something
        E = (_randn(g, V, d) * (3.0 / d ** 0.5)).bfloat16()
        target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        X = (_randn(g, T, d) + 0.8 * E[target.long()].float()).bfloat16()
        s = {"case": case, "X": X, "E": E, "w": (torch.rand(T, generator=g, device="cuda") + 0.5) / T if case["weights"] else None}
        if case["op"] == "xent":
            pos = torch.arange(T, device="cuda")
            if case["skip"] == "last":
                target = torch.where(pos % case["seq"] == case["seq"] - 1, -1, target)
            elif case["skip"] == "third":
                target = torch.where(pos % case["seq"] < case["seq"] // 3, -1, target)
            s["target"] = target.int()
            return s
        k = case["k"]
        ids = torch.randint(0, V, (T, k), generator=g, device="cuda", dtype=torch.int32)
        ids[:, 0] = target
        z = _randn(g, T, k) * 1.5 + 6.0 - 3.0 * torch.log1p(torch.arange(k, device="cuda").float())
        if case["ragged"]:  # some rows have fewer entries, some none
            n = torch.randint(0, k + 1, (T,), generator=g, device="cuda")
            ids = torch.where(torch.arange(k, device="cuda") < n[:, None], ids, -1).int()
        s["ids"], s["z"] = ids, z
        # the normaliser over the teacher's whole vocabulary: the stored entries and some mass beside them
        s["lse"] = torch.log(torch.exp(z / case["temp"]).sum(1) + 1.0 + torch.rand(T, generator=g, device="cuda")) if case["lse"] else None
        return s
    s = {"case": case, "y": (_randn(g, T, d) * 0.7 + 0.1).bfloat16(), "r": _randn(g, T, d) * 1.5 + 0.2}
    for n in ("g1", "g2"):
        s[n] = 1.0 + 0.2 * _randn(g, d)
    for n in ("b1", "b2"):
        s[n] = 0.1 * _randn(g, d) if case["shift"] else None
    rows = _gate_rows(case)
    s["gate"] = 0.5 + 0.3 * _randn(g, -(-T // rows), d) if rows else None
    if case["op"] == "norm_bwd":
        s["dh"], s["dr"] = (_randn(g, T, d) * 0.05).bfloat16(), _randn(g, T, d) * 0.05
        s["r_out"], _, s["stats"] = _plain_norm_fwd(s)
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _plain_head(s, ids, q, counted, entropy, temp):
    """ids [T, k] (any valid id where q is 0), q [T, k] targets, entropy [T] = sum q log q."""
    grad, X, E = s["case"]["grad"], s["X"].float(), s["E"].float()
    l = (X @ E.t()) / temp
    m = l.amax(1, keepdim=True)
    p = torch.exp(l - m)
    total = p.sum(1, keepdim=True)
    lse = m + torch.log(total)
    row_loss = torch.where(counted, entropy + (q * (lse - l.gather(1, ids))).sum(1), 0.0)
    w = s["w"] if s["w"] is not None else 1.0 / counted.sum().clamp(min=1)
    w = torch.where(counted, w, 0.0)
    loss = (w * row_loss).sum()
    if not grad:
        return {"loss": loss, "row_loss": row_loss, "lse": lse[:, 0]}
    p.mul_(q.sum(1, keepdim=True) / total)
    p.scatter_add_(1, ids, -q)
    p.mul_((w / temp)[:, None])
    return {"loss": loss, "row_loss": row_loss, "lse": lse[:, 0], "dX": (p @ E).bfloat16(), "dE": (p.t() @ X).bfloat16()}


def _plain_xent(s):
    counted = s["target"] >= 0
    return _plain_head(s, s["target"].clamp(min=0).long()[:, None], counted.float()[:, None], counted, torch.zeros_like(counted, dtype=torch.float32), 1.0)


def _plain_distill(s):
    temp, there = s["case"]["temp"], s["ids"] >= 0
    z = torch.where(there, s["z"] / temp, float("-inf"))
    counted = there.any(1)
    if s["lse"] is None:
        m = torch.where(counted, z.amax(1), 0.0)[:, None]
        norm = m + torch.log(torch.where(there, torch.exp(z - m), 0.0).sum(1, keepdim=True).clamp(min=1e-30))
    else:
        norm = s["lse"][:, None]
    q = torch.where(there, torch.exp(z - norm), 0.0)
    entropy = torch.where(there, q * (z - norm), 0.0).sum(1)
    return _plain_head(s, s["ids"].clamp(min=0).long(), q, counted, entropy, temp)


def _plain_norm(x, kind):
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = 1.0 / torch.sqrt(((x - mean) * (x - mean)).mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd, mean, rstd


def _rows_of(gate, case):
    """The gate of each row."""
    return 1.0 if gate is None else gate[torch.arange(case["T"], device="cuda") // _gate_rows(case)]


def _plain_norm_fwd(s):
    c = s["case"]
    yh, m1, r1 = _plain_norm(s["y"].float(), c["kind"])
    n = yh * s["g1"] + (s["b1"] if s["b1"] is not None else 0.0)
    r_out = c["scale"] * s["r"] + _rows_of(s["gate"], c) * n
    rh, m2, r2 = _plain_norm(r_out, c["kind"])
    h = rh * s["g2"] + (s["b2"] if s["b2"] is not None else 0.0)
    return r_out, h.bfloat16(), torch.cat([m1, r1, m2, r2], 1)


def _plain_norm_dx(dx_hat, x_hat, rstd, kind):
    out = dx_hat - x_hat * (dx_hat * x_hat).mean(1, keepdim=True)
    return rstd * (out - dx_hat.mean(1, keepdim=True) if kind == "layer" else out)


def _plain_norm_bwd(s):
    c, st, dh = s["case"], s["stats"], s["dh"].float()
    yh = (s["y"].float() - st[:, 0:1]) * st[:, 1:2]
    rh = (s["r_out"] - st[:, 2:3]) * st[:, 3:4]
    G = s["dr"] + _plain_norm_dx(dh * s["g2"], rh, st[:, 3:4], c["kind"])
    dn = _rows_of(s["gate"], c) * G
    out = {"dy": _plain_norm_dx(dn * s["g1"], yh, st[:, 1:2], c["kind"]).bfloat16(), "dr": c["scale"] * G,
           "dg1": (dn * yh).sum(0), "dg2": (dh * rh).sum(0)}
    if s["b1"] is not None:
        out |= {"db1": dn.sum(0), "db2": dh.sum(0)}
    if s["gate"] is not None:
        d_rows = G * (yh * s["g1"] + (s["b1"] if s["b1"] is not None else 0.0))
        out["dgate"] = torch.zeros_like(s["gate"]).index_add_(0, torch.arange(c["T"], device="cuda") // _gate_rows(c), d_rows)
    return out


# ---- the library's calls --------------------------------------------------------------------------
def _own_run(s):
    from paper_2509_22418_b200 import ppu
    c = s["case"]
    if c["op"] in ("xent", "distill"):
        if c["op"] == "xent":
            got = ppu.ppu_head_xent(s["X"], s["E"], s["target"], row_weight=s["w"], grad=c["grad"])
        else:
            got = ppu.ppu_head_distill(s["X"], s["E"], s["ids"], s["z"], temperature=c["temp"], teacher_lse=s["lse"], row_weight=s["w"], grad=c["grad"])
        names = ("loss", "row_loss", "lse", "dX", "dE")
        return {n: v for n, v in zip(names, got) if v is not None}
    more = dict(gate=s["gate"], gate_rows=_gate_rows(c), kind=c["kind"], res_scale=c["scale"])
    if c["op"] == "norm_fwd":
        r_out, h, stats = ppu.ppu_norm_gate_fwd(s["y"], s["r"], s["g1"], s["g2"], post_shift=s["b1"], pre_shift=s["b2"], eps=EPS, **more)
        return {"r_out": r_out, "h": h, "stats": stats}
    got = ppu.ppu_norm_gate_bwd(s["dh"], s["dr"], s["y"], s["r_out"], s["stats"], s["g1"], s["g2"], post_shift=s["b1"], pre_shift=s["b2"], **more)
    names = ("dy", "dr", "dg1", "db1", "dg2", "db2", "dgate")
    return {n: v for n, v in zip(names, got) if v is not None}


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "xent":
        return _plain_xent(state)
    if op == "distill":
        return _plain_distill(state)
    if op == "norm_fwd":
        r_out, h, stats = _plain_norm_fwd(state)
        return {"r_out": r_out, "h": h, "stats": stats}
    return _plain_norm_bwd(state)


def work(case):
    T, d = case["T"], case["d"]
    if case["op"] in ("xent", "distill"):
        V, k = case["V"], case.get("k", 1)
        grads = 2 if case["grad"] else 0
        # hidden states and vocabulary read, their gradients written; targets, row losses, log-sum-exps
        return {"bytes": 2 * (T + V) * d * (1 + grads // 2) + T * (8 * k + 12), "flops": 2.0 * T * V * d * (1 + grads)}
    rows = _gate_rows(case)
    gate = 4 * (-(-T // rows)) * d if rows else 0
    if case["op"] == "norm_fwd":
        return {"bytes": 12 * T * d + 16 * T + 16 * d + gate, "flops": 20.0 * T * d}
    return {"bytes": 18 * T * d + 16 * T + 32 * d + 2 * gate, "flops": 40.0 * T * d}


# ---- 64 bits, from the definitions, gradients by differentiation of the loss ---------------------
def _exact_head(s):
    c, X, E = s["case"], s["X"].double(), s["E"].double()
    T, temp = c["T"], c.get("temp", 1.0)
    if c["op"] == "xent":
        ids, there = s["target"].long()[:, None], (s["target"] >= 0)[:, None]
        q = there.double()
    else:
        ids, there = s["ids"].long(), s["ids"] >= 0
        scores = (s["z"].double() / temp).masked_fill(~there, -torch.inf)
        q = torch.exp(scores - (s["lse"].double() if c["lse"] else torch.logsumexp(scores, 1))[:, None])
        q = q.masked_fill(~there, 0.0)
    counted = there.any(1)
    w = (s["w"].double() if c["weights"] else torch.full((T,), 1.0 / max(1, int(counted.sum())), dtype=torch.float64, device="cuda")) * counted
    row_loss, lse = torch.zeros(T, dtype=torch.float64, device="cuda"), torch.zeros(T, dtype=torch.float64, device="cuda")
    dX, dE = torch.zeros_like(X) if c["grad"] else None, torch.zeros_like(E) if c["grad"] else None
    step = max(1, (1 << 27) // c["V"])
    for a in range(0, T, step):
        b = slice(a, min(T, a + step))
        logits = torch.mm(X[b], E.T).requires_grad_(c["grad"])
        full = torch.logsumexp(logits / temp, 1)
        log_p = logits.gather(1, ids[b].clamp(min=0)) / temp - full[:, None]
        rows = (torch.xlogy(q[b], q[b]) - torch.where(there[b], q[b] * log_p, 0.0)).sum(1)
        row_loss[b], lse[b] = rows.detach(), full.detach()
        if c["grad"]:
            (dl,) = torch.autograd.grad((rows * w[b]).sum(), logits)
            dX[b] = torch.mm(dl, E)
            dE += torch.mm(dl.T, X[b])
    out = {"loss": (w * row_loss).sum(), "row_loss": row_loss, "lse": lse}
    return out | ({"dX": dX, "dE": dE} if c["grad"] else {})


def _exact_norm(x, kind, eps):
    centred = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    return centred / (centred.square().mean(-1, keepdim=True) + eps).sqrt()


def _exact_pair(case, y, r, g1, b1, g2, b2, gate):
    n = _exact_norm(y, case["kind"], EPS) * g1 + b1
    if gate is not None:
        n = n * gate.repeat_interleave(_gate_rows(case), 0)[: case["T"]]
    r_out = r * case["scale"] + n
    return r_out, _exact_norm(r_out, case["kind"], EPS) * g2 + b2


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("xent", "distill"):
        return _exact_head(s)
    d = case["d"]
    zero = torch.zeros(d, dtype=torch.float64, device="cuda")
    v = [s["y"].double(), s["r"].double(), s["g1"].double(), zero.clone() if s["b1"] is None else s["b1"].double(), s["g2"].double(),
         zero.clone() if s["b2"] is None else s["b2"].double(), None if s["gate"] is None else s["gate"].double()]
    if case["op"] == "norm_fwd":
        r_out, h = _exact_pair(case, *v)
        stats = []
        for x in (v[0], r_out):
            mean = x.mean(1) if case["kind"] == "layer" else torch.zeros_like(x[:, 0])
            stats += [mean, (((x - mean[:, None]) ** 2).mean(1) + EPS).rsqrt()]
        return {"r_out": r_out, "h": h, "stats": torch.stack(stats, 1)}
    # the backward pass is given r' rounded to 32 bits: r is taken back from it, so that this is the r' differentiated at
    with torch.no_grad():
        v[1] = (s["r_out"].double() - _exact_pair({**case, "scale": 0.0}, *v)[0]) / case["scale"]
    leaves = [x.requires_grad_() for x in v if x is not None]
    r_out, h = _exact_pair(case, *v)
    got = dict(zip(("dy", "dr", "dg1", "db1", "dg2", "db2", "dgate"), torch.autograd.grad([r_out, h], leaves, [s["dr"].double(), s["dh"].double()])))
    if not case["shift"]:
        got["db1"] = got["db2"] = None
    return {n: x for n, x in got.items() if x is not None}
