"""Measured cases of the embedding pair, the query and key norms with rotation, and the orthogonalised update.

Five operators, each in a plain form of elementary torch operations (own = False) and as the
library's own call (own = True):

  embed_fwd  scaled lookup of token ids in the table
  embed_bwd  the table's gradient, alone or added to the one that the tied head has left
  qk_fwd     norm of every query and key head with its gain, rotated by position, values copied: the packed
             operand of attention from the packed product
  qk_bwd     its backward pass with the gains' gradients
  ortho      the update of matrices: momentum, then Newton-Schulz products that bring the singular values to
             about one

  embed      out_t = scale E[id_t];  dE_v = add_v + scale sum_{t: id_t = v} dout_t; negative ids are absent
  qk         y = N(x) gain for each head's x, N = x / sqrt(mean x^2 + eps) or LayerNorm; of each of the rot / 2 pairs
             (a, b) of the first rot values: (a cos - b sin, a sin + b cos), angle = position base^(-2 i / rot)
  ortho      m' = beta m + G, u = G + beta m' (without a momentum: u = G), X = u / (|u| + eps), and then 5 times
             A = X X^T, X = a X + (b A + c A A) X (for more rows than columns: of the transpose)

Sizes: the 1.3B- and 125M-class steps of this repository, and generic ragged ones around them.
"""
import torch

own = False

QK_EPS, QK_BASE = 1e-6, 10000.0
COEF, STEPS, ORTHO_EPS, BETA = (3.4445, -4.7750, 2.0315), 5, 1e-7, 0.95
LARGEST_ROWS = 8192 * 2048
LARGEST_TABLE = 32768 * 2048
LARGEST_QKV = 8192 * 6144
LARGEST_ORTHO = 3 * 2048 ** 2 * 8192 + 2048 ** 3


def listed():
    return [
        # the bottom of the 1.3B-class local step: 4 sequences of 2048 tokens into the fp32 residual stream
        {"name": "embed_fwd_step_1p3b", "op": "embed_fwd", "T": 8192, "d": 2048, "V": 32768, "ids": "zipf", "table": "bf16", "out": "fp32", "scale": 1.0},
        # one decoded token, hidden states in bf16
        {"name": "embed_fwd_one_token", "op": "embed_fwd", "T": 1, "d": 2048, "V": 32768, "ids": "uniform", "table": "bf16", "out": "bf16", "scale": 45.25},
        # the table's gradient of the 1.3B-class step, ids distributed as words are
        {"name": "embed_bwd_step_1p3b", "op": "embed_bwd", "T": 8192, "d": 2048, "V": 32768, "ids": "zipf", "dout": "fp32", "grad": "bf16", "add": False, "scale": 1.0},
        # tied table of a 125M-class model: on top of the head's gradient, padded batch, odd sizes
        {"name": "embed_bwd_tied_padded", "op": "embed_bwd", "T": 4099, "d": 768, "V": 32003, "ids": "padded", "dout": "bf16", "grad": "fp32", "add": True, "scale": 27.7},
        # attention's operand in the 1.3B-class step
        {"name": "qk_fwd_step_1p3b", "op": "qk_fwd", "T": 8192, "seq": 2048, "hq": 16, "hk": 16, "hv": 16, "dh": 128, "kind": "rms", "pairs": "adjacent", "rot": 128, "per_head": False, "far": False},
        # one decoded token far into a long text, grouped heads
        {"name": "qk_fwd_one_token_far", "op": "qk_fwd", "T": 1, "seq": 1, "hq": 32, "hk": 8, "hv": 8, "dh": 128, "kind": "rms", "pairs": "halves", "rot": 128, "per_head": False, "far": True},
        {"name": "qk_bwd_step_1p3b", "op": "qk_bwd", "T": 8192, "seq": 2048, "hq": 16, "hk": 16, "hv": 16, "dh": 128, "kind": "rms", "pairs": "adjacent", "rot": 128, "per_head": False, "far": False},
        # packed sequences with positions of their own, grouped heads of 80 of which 32 are rotated, a gain for each head
        {"name": "qk_bwd_grouped_partial", "op": "qk_bwd", "T": 1777, "seq": 301, "hq": 20, "hk": 5, "hv": 5, "dh": 80, "kind": "layer", "pairs": "halves", "rot": 32, "per_head": True, "far": True},
        # all layers' FFN slices of one replica of the 1.3B-class model (1/32: 256 hidden units)
        {"name": "ortho_slices_1p3b", "op": "ortho", "B": 24, "m": 256, "n": 2048, "grad": "fp32", "momentum": True},
        # a whole FFN matrix of it
        {"name": "ortho_ffn_1p3b", "op": "ortho", "B": 1, "m": 8192, "n": 2048, "grad": "bf16", "momentum": True},
        # the projections of the 125M-class model's layers
        {"name": "ortho_projections_125m", "op": "ortho", "B": 12, "m": 768, "n": 768, "grad": "bf16", "momentum": False},
        # one small odd matrix, where latency counts
        {"name": "ortho_small_odd", "op": "ortho", "B": 1, "m": 203, "n": 333, "grad": "fp32", "momentum": False},
    ]


def _log_int(rng, lo, hi):
    import math
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "qk_fwd", "qk_bwd", "ortho", "ortho"])
    if op in ("embed_fwd", "embed_bwd"):
        d = 8 * _log_int(rng, 1, 256)
        T = _log_int(rng, 1, min(16384, LARGEST_ROWS // d))
        V = _log_int(rng, 100, min(131072, LARGEST_TABLE // d))
        case = {"op": op, "T": T, "d": d, "V": V, "ids": rng.choice(["zipf", "uniform", "padded"]), "scale": rng.choice([1.0, 0.5, 27.7])}
        if op == "embed_fwd":
            return case | {"table": rng.choice(["bf16", "fp32"]), "out": rng.choice(["bf16", "fp32"])}
        return case | {"dout": rng.choice(["bf16", "fp32"]), "grad": rng.choice(["bf16", "fp32"]), "add": rng.random() < 0.5}
    if op in ("qk_fwd", "qk_bwd"):
        dh = 16 * _log_int(rng, 1, 16)
        hk = _log_int(rng, 1, 16)
        hq = hk * rng.choice([1, 1, 2, 4])
        T = _log_int(rng, 1, min(16384, LARGEST_QKV // ((hq + 2 * hk) * dh)))
        return {"op": op, "T": T, "seq": _log_int(rng, 1, 4096), "hq": hq, "hk": hk, "hv": rng.choice([hk, hk, 0]), "dh": dh, "kind": rng.choice(["rms", "layer"]),
                "pairs": rng.choice(["adjacent", "halves"]), "rot": rng.choice([dh, dh, 16 * rng.randint(1, dh // 16)]), "per_head": rng.random() < 0.3,
                "far": rng.random() < 0.5}
    while True:
        m, n, B = _log_int(rng, 8, 8192), _log_int(rng, 8, 8192), _log_int(rng, 1, 24)
        s, l = min(m, n), max(m, n)
        if B * s * s * (3 * l + s) <= LARGEST_ORTHO and B * s * l <= LARGEST_ROWS:
            return {"op": "ortho", "B": B, "m": m, "n": n, "grad": rng.choice(["bf16", "fp32"]), "momentum": rng.random() < 0.5}


# ---- inputs -------------------------------------------------------------------------------------
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _ids(case, g):
    T, V = case["T"], case["V"]
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    if case["ids"] == "uniform":
        ids = (u * V).long()
    else:  # frequency falling about as 1 / rank, the ranks spread over the table
        rank = torch.exp(u * torch.log(torch.tensor(V + 1.0, dtype=torch.float64, device="cuda"))).long() - 1
        ids = (rank * 7919) % V
    ids = ids.clamp(0, V - 1)
    if case["ids"] == "padded":  # the ends of sequences
        t = torch.arange(T, device="cuda")
        ids = torch.where(t % 512 >= 400, -1, ids)
    return ids.int()


def _gradient(g, B, m, n):
    """A product of hidden states and their gradients over tokens, a few directions of which carry most."""
    k = max(1, min(m, n) // 4)
    fall = torch.arange(1, k + 1, device="cuda").float() ** -0.5
    out = torch.matmul(_randn(g, B, m, k) * fall, _randn(g, B, k, n))
    return 1e-3 * (out + 0.3 * _randn(g, B, m, n))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op in ("embed_fwd", "embed_bwd"):
        T, d, V = case["T"], case["d"], case["V"]
        s["ids"] = _ids(case, g)
        if op == "embed_fwd":
            s["E"] = (0.02 * _randn(g, V, d)).to(_TYPES[case["table"]])
        else:
            s["dout"] = (1e-3 * _randn(g, T, d)).to(_TYPES[case["dout"]])
            s["add"] = (1e-3 * _randn(g, V, d)).to(_TYPES[case["grad"]]) if case["add"] else None
        return s
    if op in ("qk_fwd", "qk_bwd"):
        T, dh, hq, hk = case["T"], case["dh"], case["hq"], case["hk"]
        s["qkv"] = _randn(g, T, (hq + hk + case["hv"]) * dh).bfloat16()
        s["q_gain"], s["k_gain"] = (1.0 + 0.2 * _randn(g, *((h, dh) if case["per_head"] else (dh,))) for h in (hq, hk))
        # positions of their own: sequences that begin somewhere in a long text
        start = torch.randint(0, 1 << 20, (-(-T // case["seq"]),), generator=g, device="cuda")
        t = torch.arange(T, device="cuda")
        s["positions"] = (t % case["seq"] + start[t // case["seq"]]).int() if case["far"] else None
        if op == "qk_bwd":
            s["dout"] = (0.05 * _randn(g, *s["qkv"].shape)).bfloat16()
        return s
    B, m, n = case["B"], case["m"], case["n"]
    s["G"] = _gradient(g, B, m, n).to(_TYPES[case["grad"]])
    s["momentum"] = 5.0 * _gradient(g, B, m, n) if case["momentum"] else None
    return s


# ---- plain forms ----------------------------------------------------------------------------------
def _plain_embed_fwd(s):
    c, ids = s["case"], s["ids"].long()
    rows = s["E"][ids.clamp(min=0)].float() * c["scale"]
    return {"out": torch.where(ids[:, None] >= 0, rows, 0.0).to(_TYPES[c["out"]])}


def _plain_embed_bwd(s):
    c, ids = s["case"], s["ids"].long()
    there = ids >= 0
    dE = torch.zeros((c["V"], c["d"]), dtype=torch.float32, device="cuda")
    dE.index_add_(0, ids.clamp(min=0), torch.where(there[:, None], s["dout"].float() * c["scale"], 0.0))
    if s["add"] is not None:
        dE += s["add"].float()
    return {"dE": dE.to(_TYPES[c["grad"]])}


def _plain_angles(s):
    """cos, sin [T, 1, rot / 2], of angles formed in 64 bits: positions go far."""
    c = s["case"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(c["T"], device="cuda") % c["seq"]
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    angle = pos.double()[:, None, None] * torch.exp(i * (-2.0 / c["rot"]) * torch.log(torch.tensor(QK_BASE, dtype=torch.float64, device="cuda")))
    return torch.cos(angle).float(), torch.sin(angle).float()


def _plain_rotate(x, c, cos, sin):
    r = c["rot"]
    if c["pairs"] == "adjacent":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        out = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        out = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([out, x[..., r:]], -1)


def _plain_head_norm(x, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + QK_EPS)
    return x * rstd, rstd


def _heads(t, c):
    """[T, heads, dh] views of the queries, keys and values of a packed operand."""
    return t.view(c["T"], -1, c["dh"]).split([c["hq"], c["hk"], c["hv"]], 1)


def _plain_qk_fwd(s):
    c = s["case"]
    cos, sin = _plain_angles(s)
    q, k, v = _heads(s["qkv"], c)
    out = [_plain_rotate(_plain_head_norm(x.float(), c["kind"])[0] * gain, c, cos, sin).bfloat16() for x, gain in ((q, s["q_gain"]), (k, s["k_gain"]))]
    return {"qkv": torch.cat(out + [v], 1).flatten(1)}


def _plain_qk_bwd(s):
    c = s["case"]
    cos, sin = _plain_angles(s)
    out, grads = [], {}
    (q, k, _), (dq, dk, dv) = _heads(s["qkv"], c), _heads(s["dout"], c)
    for name, x, dy, gain in (("q_gain", q, dq, s["q_gain"]), ("k_gain", k, dk, s["k_gain"])):
        xh, rstd = _plain_head_norm(x.float(), c["kind"])
        g = _plain_rotate(dy.float(), c, cos, -sin)
        grads["d" + name] = (g * xh).sum(0) if c["per_head"] else (g * xh).sum((0, 1))
        w = g * gain
        dx = w - xh * (w * xh).mean(-1, keepdim=True)
        if c["kind"] == "layer":
            dx = dx - w.mean(-1, keepdim=True)
        out.append((rstd * dx).bfloat16())
    return {"dqkv": torch.cat(out + [dv], 1).flatten(1), **grads}


def _plain_ortho(s):
    u, new = s["G"].float(), None
    if s["momentum"] is not None:
        new = BETA * s["momentum"] + u
        u = u + BETA * new
    tall = u.shape[1] > u.shape[2]
    X = u.transpose(1, 2) if tall else u
    X = X / (torch.sqrt((X.double() * X.double()).sum((1, 2), keepdim=True)) + ORTHO_EPS).float()
    for _ in range(STEPS):
        A = torch.matmul(X, X.transpose(1, 2))
        X = COEF[0] * X + torch.matmul(COEF[1] * A + COEF[2] * torch.matmul(A, A), X)
    out = {"O": (X.transpose(1, 2) if tall else X).bfloat16().contiguous()}
    return out if new is None else out | {"momentum": new}


# ---- the library's calls --------------------------------------------------------------------------
def _own_run(s):
    from paper_2509_22418_b200 import ppu
    c = s["case"]
    if c["op"] == "embed_fwd":
        return {"out": ppu.ppu_embed_fwd(s["ids"], s["E"], scale=c["scale"], dtype=c["out"])}
    if c["op"] == "embed_bwd":
        return {"dE": ppu.ppu_embed_bwd(s["ids"], s["dout"], c["V"], scale=c["scale"], dtype=c["grad"], add=s["add"])}
    if c["op"] in ("qk_fwd", "qk_bwd"):
        more = dict(q_gain=s["q_gain"], k_gain=s["k_gain"], positions=s["positions"], seq=c["seq"], kind=c["kind"], eps=QK_EPS, rope_base=QK_BASE,
                    rot_dim=c["rot"], pairs=c["pairs"])
        if c["op"] == "qk_fwd":
            return {"qkv": ppu.ppu_qk_norm_fwd(s["qkv"], c["hq"], c["hk"], c["hv"], **more)}
        return dict(zip(("dqkv", "dq_gain", "dk_gain"), ppu.ppu_qk_norm_bwd(s["dout"], s["qkv"], c["hq"], c["hk"], c["hv"], **more)))
    O, new = ppu.ppu_orthogonalize(s["G"], momentum=s["momentum"], beta=BETA, nesterov=True, steps=STEPS, coef=COEF, eps=ORTHO_EPS)
    return {"O": O} if new is None else {"O": O, "momentum": new}


_PLAIN = {"embed_fwd": _plain_embed_fwd, "embed_bwd": _plain_embed_bwd, "qk_fwd": _plain_qk_fwd, "qk_bwd": _plain_qk_bwd, "ortho": _plain_ortho}


def run(state):
    return _own_run(state) if own else _PLAIN[state["case"]["op"]](state)


def _bytes(word):
    return 2 if word == "bf16" else 4


def work(case):
    op = case["op"]
    if op in ("embed_fwd", "embed_bwd"):
        T, d, V = case["T"], case["d"], case["V"]
        if op == "embed_fwd":  # rows of the table read once each at most
            return {"bytes": min(T, V) * d * _bytes(case["table"]) + T * d * _bytes(case["out"]) + 4 * T, "flops": 1.0 * T * d}
        return {"bytes": T * d * _bytes(case["dout"]) + V * d * _bytes(case["grad"]) * (2 if case["add"] else 1) + 4 * T, "flops": 2.0 * T * d}
    if op in ("qk_fwd", "qk_bwd"):
        T, dh, h, hv = case["T"], case["dh"], case["hq"] + case["hk"], case["hv"]
        gains = 4 * dh * (h if case["per_head"] else 2)
        if op == "qk_fwd":
            return {"bytes": 4 * T * (h + hv) * dh + gains + (4 * T if case["far"] else 0), "flops": 8.0 * T * h * dh}
        return {"bytes": 6 * T * h * dh + 4 * T * hv * dh + 2 * gains + (4 * T if case["far"] else 0), "flops": 16.0 * T * h * dh}
    B, s, l = case["B"], min(case["m"], case["n"]), max(case["m"], case["n"])
    # A and A A are symmetric: half of each
    return {"bytes": B * s * l * (_bytes(case["grad"]) + 2 + (8 if case["momentum"] else 0)), "flops": 1.0 * STEPS * B * s * s * (3 * l + s)}


# ---- 64 bits, from the definitions, gradients by differentiation ----------------------------------
def _exact_qk(x, gains, c, positions):
    """x [T, heads, dh] of queries and keys; as complex numbers turned by exp(i angle)."""
    eps = QK_EPS
    if c["kind"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * gains
    r = c["rot"]
    freq = QK_BASE ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(c["T"], r // 2), positions[:, None] * freq)[:, None]
    head, rest = y[..., :r], y[..., r:]
    if c["pairs"] == "adjacent":
        z = torch.view_as_complex(head.unflatten(-1, (r // 2, 2)).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(head[..., : r // 2], head[..., r // 2:]) * turn
        head = torch.cat([z.real, z.imag], -1)
    return torch.cat([head, rest], -1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed_fwd":
        table = torch.cat([s["E"].double(), torch.zeros((1, case["d"]), dtype=torch.float64, device="cuda")])
        return {"out": table[torch.where(s["ids"] < 0, case["V"], s["ids"]).long()] * case["scale"]}
    if op == "embed_bwd":
        dE = torch.zeros((case["V"] + 1, case["d"]), dtype=torch.float64, device="cuda")
        dE.index_add_(0, torch.where(s["ids"] < 0, case["V"], s["ids"]).long(), s["dout"].double())
        dE = dE[:-1] * case["scale"]
        return {"dE": dE if s["add"] is None else dE + s["add"].double()}
    if op in ("qk_fwd", "qk_bwd"):
        T, h = case["T"], case["hq"] + case["hk"]
        packed = s["qkv"].double().view(T, -1, case["dh"])
        x = packed[:, :h].clone().requires_grad_()
        gq, gk = s["q_gain"].double().requires_grad_(), s["k_gain"].double().requires_grad_()
        gains = torch.cat([gq.expand(case["hq"], -1), gk.expand(case["hk"], -1)])
        pos = (s["positions"] if case["far"] else torch.arange(T, device="cuda") % case["seq"]).double()
        y = _exact_qk(x, gains, case, pos)
        if op == "qk_fwd":
            return {"qkv": torch.cat([y.detach(), packed[:, h:]], 1).flatten(1)}
        dout = s["dout"].double().view(T, -1, case["dh"])
        dx, dgq, dgk = torch.autograd.grad(y, [x, gq, gk], dout[:, :h].contiguous())
        return {"dqkv": torch.cat([dx, dout[:, h:]], 1).flatten(1), "dq_gain": dgq, "dk_gain": dgk}
    u, new = s["G"].double(), None
    if case["momentum"]:
        new = s["momentum"].double() * BETA + u
        u = u + new * BETA
    a, b, c = COEF
    X = u / (torch.linalg.matrix_norm(u, keepdim=True) + ORTHO_EPS)
    tall = case["m"] > case["n"]
    eye = torch.eye(min(case["m"], case["n"]), dtype=torch.float64, device="cuda")
    for _ in range(STEPS):
        A = X.mT @ X if tall else X @ X.mT
        Q = a * eye + A @ (b * eye + c * A)
        X = X @ Q if tall else Q @ X
    return {"O": X} if new is None else {"O": X, "momentum": new}
