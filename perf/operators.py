"""Cases of the operators around the policy's logits and its update, each in a plain form too.

``logits``       pace.logits_logprob: log-probs of given tokens, entropy and top
                 alternatives from logits in memory (a rollout engine's decode step,
                 a batch that is re-scored).
``logits_grad``  pace.logits_logprob_backward: the gradient of log-probs and entropies
                 with respect to the logits.
``head``         pace.token_logprob_entropy: log-probs and entropies through the fused
                 LM head, logits never in memory.
``head_grad``    pace.token_logprob_entropy_backward: gradients of hidden states and of
                 the vocabulary matrix, in bf16.
``ortho``        pace.orthogonalize: Newton-Schulz products on a stack of updates.
``muon``         pace.muon_update: momentum, orthogonalised update, weight decay.

``own`` selects the framework's calls; otherwise ``run`` computes the plain forms:
elementary torch operations in 32 bits.  Shapes: the hidden sizes and vocabularies are
those of the package's workloads (256 / 2,048; 1,024 / 50,001; 2,048 / 151,936; 3,584 /
152,064) and multiples of them.
"""
import math

import torch

own = False

DEV = "cuda"
F16, BF16, F32, F64 = torch.float16, torch.bfloat16, torch.float32, torch.float64
I32, I64, U8 = torch.int32, torch.int64, torch.uint8
DTYPES = {"f16": F16, "bf16": BF16, "f32": F32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
NS_STEPS, NS_COEF, NS_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # A decode step of four sequences: log-prob of the sampled token, entropy and
        # twenty alternatives.  Latency of one call.
        {"name": "decode_top20", "op": "logits", "rows": 4, "V": 151936, "dtype": "bf16",
         "top": 20, "tau": 1.0, "allowed": False, "pad": 0},
        # Re-scoring a batch whose logits are in memory, an odd number of rows.
        {"name": "rescore_4099", "op": "logits", "rows": 4099, "V": 151936, "dtype": "bf16",
         "top": 5, "tau": 0.7, "allowed": False, "pad": 0},
        # A constrained decode batch: fp32 logits in a padded buffer, odd vocabulary, a
        # bit per place that the grammar allows, one row of which nothing is left; gradient.
        {"name": "grad_constrained_97", "op": "logits_grad", "rows": 97, "V": 50001,
         "dtype": "f32", "tau": 0.7, "allowed": True, "pad": 3, "entropy": True},
        # Gradient of a whole micro-batch's logits.
        {"name": "grad_batch_2583", "op": "logits_grad", "rows": 2583, "V": 151936,
         "dtype": "bf16", "tau": 1.0, "allowed": False, "pad": 0, "entropy": True},
        # The fused head on the tokens of one decode step: the vocabulary matrix is read
        # for a handful of rows.
        {"name": "head_8_rows", "op": "head", "n_seq": 8, "len": 1, "prompt": 0, "H": 2048,
         "V": 151936, "tau": 1.0},
        # A micro-batch on the 7B-shaped head with its prompts masked out.
        {"name": "head_batch", "op": "head", "n_seq": 8, "len": 256, "prompt": 64, "H": 3584,
         "V": 152064, "tau": 1.0},
        # Gradients on a small model's head, an odd vocabulary, ragged sequences.
        {"name": "head_grad_small", "op": "head_grad", "n_seq": 5, "len": 61, "prompt": 7,
         "H": 1024, "V": 50001, "tau": 0.7, "entropy": True},
        # Gradients of one micro-batch.
        {"name": "head_grad_batch", "op": "head_grad", "n_seq": 8, "len": 256, "prompt": 64,
         "H": 2048, "V": 151936, "tau": 1.0, "entropy": True},
        # One small layer's update.
        {"name": "ortho_256", "op": "ortho", "batch": 1, "m": 256, "n": 256, "dtype": "bf16"},
        # Updates of three layers at once, tall, with an odd width.
        {"name": "ortho_2731x1023_x3", "op": "ortho", "batch": 3, "m": 2731, "n": 1023,
         "dtype": "f32"},
        # The whole step on a square attention projection.
        {"name": "muon_2048", "op": "muon", "batch": 1, "m": 2048, "n": 2048, "dtype": "f32",
         "nesterov": True},
        # The whole step on the largest matrix of a block.
        {"name": "muon_3584x14336", "op": "muon", "batch": 1, "m": 3584, "n": 14336,
         "dtype": "bf16", "nesterov": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("logits", "logits", "logits_grad", "head", "head_grad", "ortho", "muon"))
    if op in ("logits", "logits_grad"):
        V = rng.choice((2048, 50001, 151936, 152064, _log_int(rng, 500, 151936)))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        most = 4099 if op == "logits" else 2583
        rows = _log_int(rng, 1, most if dtype != "f32" else most // 2)
        c = {"op": op, "rows": rows, "V": V, "dtype": dtype, "tau": rng.choice((1.0, 0.7, 1.3)),
             "allowed": rng.random() < 0.4, "pad": rng.choice((0, 0, 1, 8, 61))}
        if op == "logits":
            c["top"] = rng.choice((0, 1, 5, 20, rng.randint(2, 64)))
        else:
            c["entropy"] = rng.random() < 0.6
        return c
    if op in ("head", "head_grad"):
        H, V = rng.choice(((256, 2048), (1024, 50001), (2048, 151936), (3584, 152064),
                           (64 * rng.randint(2, 32), _log_int(rng, 1000, 100000))))
        if op == "head_grad" and H > 2048:
            H, V = 2048, 151936
        c = {"op": op, "n_seq": rng.randint(1, 8), "len": _log_int(rng, 1, 256),
             "prompt": rng.choice((0, rng.randint(1, 64))), "H": H, "V": V,
             "tau": rng.choice((1.0, 0.7))}
        if op == "head_grad":
            c["entropy"] = rng.random() < 0.6
        return c
    while True:
        m, n, batch = _log_int(rng, 32, 4096), _log_int(rng, 32, 14336), rng.choice((1, 1, 2, 6))
        if batch * _ns_flops(m, n) <= _ns_flops(3584, 14336):
            break
    c = {"op": op, "batch": batch, "m": m, "n": n, "dtype": rng.choice(("bf16", "f32"))}
    if op == "muon":
        c["nesterov"] = rng.random() < 0.7
    return c


# ------------------------------------------------------------------ the inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rand(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _randint(g, lo, hi, n):
    return torch.randint(lo, hi, (n,), generator=g, device=DEV, dtype=I32)


def _rows_of(case):
    """Rows of a logits case that are in the loss: nine of ten in the gradient cases."""
    return case["op"] == "logits_grad"


def _prepare_logits(case, seed):
    g = _gen(seed)
    R, V, dt = case["rows"], case["V"], DTYPES[case["dtype"]]
    # logits of a language model: spread 2, with one place in a hundred lifted to where the
    # likely tokens are; the row's pitch may be larger than the vocabulary
    buf = torch.empty((R, V + case["pad"]), dtype=dt, device=DEV)
    for i in range(0, R, 512):
        part = _rand(g, min(512, R - i), V + case["pad"]) * 2
        part += 6 * (torch.rand(part.shape, generator=g, device=DEV) < 0.01)
        buf[i:i + 512] = part.to(dt)
    s = {"case": case, "kept": {}, "logits": buf[:, :V], "targets": _randint(g, 0, V, R)}
    s["allowed"] = s["mask"] = None
    if case["allowed"]:
        words = (V + 31) // 32
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (R, words), generator=g, device=DEV,
                                     dtype=I64).to(I32)
        s["allowed"][R // 2] = 0  # a row of which nothing is left
    if _rows_of(case):
        s["mask"] = (torch.rand(R, generator=g, device=DEV) < 0.9).to(U8)
        s["dlp"] = _rand(g, R) / R
        s["dent"] = _rand(g, R) * (0.01 / R) if case["entropy"] else None
        s["stats"], s["entropy"] = _row_stats(s)
    return s


def _allowed_places(s, rows):
    """bool [rows, V] of the places that the bits allow."""
    V = s["case"]["V"]
    j = torch.arange(V, device=DEV)
    return (s["allowed"][rows][:, j // 32] >> (j % 32) & 1).bool()


def _row_stats(s):
    """What the forward leaves for the backward: (largest logit, ln of the sum) and entropy."""
    R, tau = s["case"]["rows"], s["case"]["tau"]
    stats, ent = torch.empty((R, 2), device=DEV), torch.empty(R, device=DEV)
    for i in range(0, R, 256):
        rows = slice(i, min(R, i + 256))
        z = s["logits"][rows].float()
        if s["allowed"] is not None:
            z = torch.where(_allowed_places(s, rows), z, -math.inf)
        m = z.amax(1)
        d = (z - torch.where(m > -math.inf, m, 0 * m)[:, None]) / tau
        e = torch.exp(d)
        total = e.sum(1)
        h = torch.log(total) - torch.where(e > 0, e * d, 0 * e).sum(1) / total
        stats[rows, 0], stats[rows, 1] = m, torch.log(total)
        ent[rows] = torch.where(total > 0, h, 0 * h)
    keep = s["mask"] > 0
    return torch.where(keep[:, None], stats, 0 * stats.nan_to_num()), torch.where(keep, ent, 0 * ent)


def _prepare_head(case, seed):
    g = _gen(seed)
    n, H, V, tau = case["n_seq"], case["H"], case["V"], case["tau"]
    # ragged responses around the stated length, after a prompt that is not in the loss
    lens = [max(1, case["len"] + (17 * i + 5) % 23 - 11) if case["len"] > 16 else case["len"]
            for i in range(n)]
    seg = torch.tensor([x for k in lens for x in (case["prompt"], k)])
    mask = torch.repeat_interleave(torch.tensor([0, 1], dtype=U8).repeat(n), seg).to(DEV)
    offsets = torch.cat([torch.zeros(1, dtype=I64), torch.cumsum(seg.reshape(n, 2).sum(1), 0)])
    R = mask.numel()
    s = {"case": case, "kept": {}, "mask": mask, "offsets": offsets.to(DEV),
         "in_loss": mask.nonzero()[:, 0], "hidden": _rand(g, R, H, dtype=BF16),
         "w": _rand(g, V, H, dtype=BF16).mul_(2.0 / math.sqrt(H)),
         "targets": _randint(g, 0, V, R)}
    if case["op"] == "head_grad":
        z = _head_logits(s)
        lse, ent = torch.zeros(R, device=DEV), torch.zeros(R, device=DEV)
        lse[s["in_loss"]] = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        ent[s["in_loss"]] = lse[s["in_loss"]] - (p * z).sum(1)
        s["lse"], s["entropy"] = lse, ent
        s["dlp"] = _rand(g, R) / R * mask
        s["dent"] = _rand(g, R) * (0.05 / R) * mask if case["entropy"] else None
    return s


def _head_logits(s, dtype=F32):
    z = s["hidden"][s["in_loss"]].to(dtype) @ s["w"].to(dtype).T
    return z.div_(s["case"]["tau"])


def _prepare_matrix(case, seed):
    g = _gen(seed)
    B, m, n, dt = case["batch"], case["m"], case["n"], DTYPES[case["dtype"]]
    # a layer's gradient: a few strong directions on a broad floor, at a gradient's scale
    r = max(1, min(m, n) // 16)
    u = _rand(g, B, m, r) @ _rand(g, B, r, n) / math.sqrt(r) + _rand(g, B, m, n)
    s = {"case": case, "kept": {}, "x": (u * 1e-4).to(dt)}
    if case["op"] == "muon":
        s["momentum"] = _rand(g, B, m, n) * 5e-4
        s["weight"] = _rand(g, B, m, n) / math.sqrt(n)
        s["copy"] = torch.empty((B, m, n), dtype=BF16, device=DEV)
    return s


MUON = {"lr": 2e-5, "mu": 0.95, "decay": 0.1}


def _muon_scale(case):
    """Updates of the same root mean square whatever the matrix's shape."""
    return 0.2 * math.sqrt(max(case["m"], case["n"]))


def prepare(case, seed):
    if case["op"] in ("logits", "logits_grad"):
        return _prepare_logits(case, seed)
    if case["op"] in ("head", "head_grad"):
        return _prepare_head(case, seed)
    return _prepare_matrix(case, seed)


# ------------------------------------------------------------------ the plain forms

def _first_of(values, k):
    """Indices of the k largest values of each row, ties to the lowest index."""
    V = values.shape[1]
    bits = (values + 0.0).view(I32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(I64)
    key = order * 2 ** 32 + (V - 1 - torch.arange(V, device=DEV))
    return V - 1 - (torch.topk(key, min(k, V), dim=1).values & 0xFFFFFFFF)


def _plain_logits(s):
    c = s["case"]
    tau, k = c["tau"], c["top"]
    z = s["logits"].float()
    if s["allowed"] is not None:
        z = torch.where(_allowed_places(s, slice(None)), z, -math.inf)
    m = z.amax(1, keepdim=True)
    empty = m[:, 0] == -math.inf
    d = (z - torch.where(m > -math.inf, m, 0 * m)) / tau
    e = torch.exp(d)
    total = e.sum(1)
    log_s = torch.log(total)
    dy = d.gather(1, s["targets"].to(I64)[:, None])[:, 0]
    none = torch.full_like(log_s, -math.inf)
    out = {"logprob": torch.where(empty, none, dy - log_s),
           "lse": torch.where(empty, none, m[:, 0] / tau + log_s),
           "entropy": torch.where(empty, 0 * total,
                                  log_s - torch.where(e > 0, e * d, 0 * e).sum(1) / total)}
    if k:
        ids = _first_of(z, k)
        top = d.gather(1, ids) - log_s[:, None]
        there = z.gather(1, ids) > -math.inf
        out["top_ids"] = torch.where(there, ids, -1).to(I32)
        out["top_logprob"] = torch.where(there, top, torch.full_like(top, -math.inf))
    return out


def _plain_logits_grad(s):
    c = s["case"]
    tau, m, log_s = c["tau"], s["stats"][:, :1], s["stats"][:, 1:]
    z = s["logits"].float()
    if s["allowed"] is not None:
        z = torch.where(_allowed_places(s, slice(None)), z, -math.inf)
    lp = (z - m) / tau - log_s
    p = torch.exp(lp)
    grad = -s["dlp"][:, None] * p
    if s["dent"] is not None:
        grad -= s["dent"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0 * p)
    y = s["targets"].to(I64)[:, None]
    hit = grad.gather(1, y) + s["dlp"][:, None]
    grad.scatter_(1, y, hit)
    live = (s["mask"] > 0)[:, None] & (m > -math.inf) & (z > -math.inf)
    return torch.where(live, grad / tau, torch.zeros_like(z)).to(DTYPES[c["dtype"]])


def _plain_head(s):
    z = _head_logits(s)
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1)
    y = s["targets"][s["in_loss"]].to(I64)[:, None]
    out = {}
    for name, v in (("logprob", d.gather(1, y)[:, 0] - torch.log(total)),
                    ("lse", m[:, 0] + torch.log(total)),
                    ("entropy", torch.log(total) - (e * d).sum(1) / total)):
        out[name] = torch.zeros(s["mask"].numel(), device=DEV)
        out[name][s["in_loss"]] = v
    return out


def _head_grad(s, dtype):
    """(dH, dW) in `dtype` from its products."""
    at = s["in_loss"]
    lp = _head_logits(s, dtype) - s["lse"][at].to(dtype)[:, None]
    p = torch.exp(lp)
    g = -s["dlp"][at].to(dtype)[:, None] * p
    if s["dent"] is not None:
        g -= s["dent"][at].to(dtype)[:, None] * p * (lp + s["entropy"][at].to(dtype)[:, None])
    y = s["targets"][at].to(I64)[:, None]
    g.scatter_add_(1, y, s["dlp"][at].to(dtype)[:, None])
    g /= s["case"]["tau"]
    dh = torch.zeros((s["mask"].numel(), s["case"]["H"]), dtype=dtype, device=DEV)
    dh[at] = g @ s["w"].to(dtype)
    return dh, g.T @ s["hidden"][at].to(dtype)


def _newton_schulz(u):
    """The Newton-Schulz steps on a stack of matrices, in the type of u."""
    a, b, c = NS_COEF
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _muon(case, x, momentum, weight, dtype):
    """The new (momentum, weight) in `dtype`."""
    g = x.to(dtype)
    momentum = MUON["mu"] * momentum.to(dtype) + g
    u = g + MUON["mu"] * momentum if case["nesterov"] else momentum
    o = _newton_schulz(u)
    weight = weight.to(dtype) * (1 - MUON["lr"] * MUON["decay"])
    return momentum, weight - MUON["lr"] * _muon_scale(case) * o


def _plain(s):
    op = s["case"]["op"]
    if op == "logits":
        return _plain_logits(s)
    if op == "logits_grad":
        return {"grad": _plain_logits_grad(s)}
    if op == "head":
        return _plain_head(s)
    if op == "head_grad":
        dh, dw = _head_grad(s, F32)
        return {"grad_hidden": dh.to(BF16), "grad_w": dw.to(BF16)}
    if op == "ortho":
        return {"update": _newton_schulz(s["x"].float()).to(BF16)}
    momentum, weight = _muon(s["case"], s["x"], s["momentum"], s["weight"], F32)
    s["momentum"].copy_(momentum)
    s["weight"].copy_(weight)
    s["copy"].copy_(weight)
    return {"momentum": s["momentum"], "weight": s["weight"], "weight_bf16": s["copy"]}


# ------------------------------------------------------------------ the framework's calls

def _keep(s, pace):
    """Outputs, workspaces and descriptions that a program allocates once for its shape."""
    c, k = s["case"], s["kept"]
    k["status"] = pace.new_status(DEV)
    if c["op"] in ("logits", "logits_grad"):
        k["lg"] = pace.make_logits(s["logits"], allowed=s["allowed"], mask=s["mask"])
        if c["op"] == "logits":
            k["out"] = pace.logits_logprob_outputs(c["rows"], c["top"], DEV)
        else:
            k["grad"] = torch.empty((c["rows"], c["V"]), dtype=DTYPES[c["dtype"]], device=DEV)
    elif c["op"] in ("head", "head_grad"):
        R, H, V = s["mask"].numel(), c["H"], c["V"]
        k["batch"] = pace.make_batch(s["offsets"], R, mask=s["mask"])
        if c["op"] == "head":
            k["out"] = {n: torch.empty(R, device=DEV) for n in ("logprob", "lse", "entropy")}
            size = pace.token_logprob_entropy_workspace_size(R, c["n_seq"], H, V)
        else:
            k["gh"] = torch.empty((R, H), dtype=BF16, device=DEV)
            k["gw"] = torch.empty((V, H), dtype=BF16, device=DEV)
            size = pace.token_logprob_entropy_backward_workspace_size(R, c["n_seq"], H, V, BF16)
        k["ws"] = pace.workspace(size, DEV)
    else:
        k["ws"] = pace.workspace(pace.muon_workspace_size(c["batch"], c["m"], c["n"]), DEV)
        if c["op"] == "ortho":
            k["out"] = torch.empty(s["x"].shape, dtype=BF16, device=DEV)
            k["params"] = pace.muon_params(steps=NS_STEPS, coef=NS_COEF, eps=NS_EPS)
        else:
            k["params"] = pace.muon_params(
                lr=MUON["lr"], momentum=MUON["mu"], weight_decay=MUON["decay"],
                nesterov=c["nesterov"], scale=_muon_scale(c), steps=NS_STEPS, coef=NS_COEF,
                eps=NS_EPS)


def _own(s):
    from paper_2609_36830_gb300 import pace
    c, k = s["case"], s["kept"]
    if not k:
        _keep(s, pace)
    if c["op"] == "logits":
        o = pace.logits_logprob(k["lg"], s["targets"], temperature=c["tau"], top_k=c["top"],
                                out=k["out"], status=k["status"])
        names = ("logprob", "lse", "entropy") + (("top_ids", "top_logprob") if c["top"] else ())
        return {n: o[n] for n in names}
    if c["op"] == "logits_grad":
        return {"grad": pace.logits_logprob_backward(
            k["lg"], s["targets"], s["stats"], s["dlp"], entropy=s["entropy"],
            dentropy=s["dent"], temperature=c["tau"], grad=k["grad"], status=k["status"])}
    if c["op"] == "head":
        o = k["out"]
        pace.token_logprob_entropy(k["batch"], s["hidden"], s["w"], s["targets"], c["tau"],
                                   logprob=o["logprob"], lse=o["lse"], entropy=o["entropy"],
                                   ws=k["ws"], status=k["status"])
        return o
    if c["op"] == "head_grad":
        gh, gw = pace.token_logprob_entropy_backward(
            k["batch"], s["hidden"], s["w"], s["targets"], s["lse"], s["dlp"],
            entropy=s["entropy"], dentropy=s["dent"], temperature=c["tau"], grad_hidden=k["gh"],
            grad_w=k["gw"], ws=k["ws"], status=k["status"])
        return {"grad_hidden": gh, "grad_w": gw}
    if c["op"] == "ortho":
        return {"update": pace.orthogonalize(s["x"], k["params"], out=k["out"], ws=k["ws"],
                                             status=k["status"])}
    pace.muon_update(s["weight"], s["x"], s["momentum"], k["params"], weight_bf16=s["copy"],
                     ws=k["ws"], status=k["status"])
    return {"momentum": s["momentum"], "weight": s["weight"], "weight_bf16": s["copy"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ floors and 64-bit results

def _ns_flops(m, n):
    """The products of the Newton-Schulz steps, each symmetric one by its half."""
    s, l = min(m, n), max(m, n)
    return NS_STEPS * (3.0 * s * s * l + float(s) ** 3)


def _rows_in_loss(case):
    return sum(max(1, case["len"] + (17 * i + 5) % 23 - 11) if case["len"] > 16 else case["len"]
               for i in range(case["n_seq"]))


def work(case):
    op = case["op"]
    if op in ("logits", "logits_grad"):
        n = float(case["rows"]) * case["V"]
        moved = n * BYTES[case["dtype"]] + (n / 8 if case["allowed"] else 0)
        if op == "logits":
            return {"bytes": moved + case["rows"] * (16 + 8 * case["top"]), "flops": 6 * n}
        return {"bytes": moved + n * BYTES[case["dtype"]] + 24 * case["rows"], "flops": 8 * n}
    if op in ("head", "head_grad"):
        R, H, V = _rows_in_loss(case), case["H"], case["V"]
        once = 2.0 * (R * H + V * H)
        if op == "head":
            return {"bytes": once + 16 * R, "flops": 2.0 * R * H * V}
        return {"bytes": 2 * once + 20 * R, "flops": 6.0 * R * H * V}
    B, size = case["batch"], float(case["batch"]) * case["m"] * case["n"]
    flops = B * _ns_flops(case["m"], case["n"])
    if op == "ortho":
        return {"bytes": size * (BYTES[case["dtype"]] + 2), "flops": flops}
    return {"bytes": size * (BYTES[case["dtype"]] + 8 + 8 + 2), "flops": flops}


def _exact_logits(s):
    c = s["case"]
    R, V, tau, k = c["rows"], c["V"], c["tau"], c["top"]
    out = {n: torch.empty(R, dtype=F64, device=DEV) for n in ("logprob", "lse", "entropy")}
    top = torch.full((R, min(k, V)), -math.inf, dtype=F64, device=DEV)
    for i in range(0, R, 128):
        rows = slice(i, min(R, i + 128))
        z = s["logits"][rows].to(F64) / tau
        if s["allowed"] is not None:
            z[~_allowed_places(s, rows)] = -math.inf
        lse = torch.logsumexp(z, 1)
        lp = z - lse[:, None]
        lp[lse == -math.inf] = -math.inf
        p = torch.exp(lp)
        out["lse"][rows] = lse
        out["logprob"][rows] = lp.gather(1, s["targets"][rows].to(I64)[:, None])[:, 0]
        out["entropy"][rows] = -torch.where(p > 0, p * lp, 0 * p).sum(1)
        if k:
            top[rows] = torch.topk(lp, min(k, V), dim=1).values
    if k:
        out.update(top_ids=None, top_logprob=top)
    return out


def _exact_logits_grad(s):
    c = s["case"]
    R, V, tau = c["rows"], c["V"], c["tau"]
    out = torch.zeros((R, V), dtype=F64, device=DEV)
    for i in range(0, R, 128):
        rows = slice(i, min(R, i + 128))
        z = s["logits"][rows].to(F64)
        if s["allowed"] is not None:
            z[~_allowed_places(s, rows)] = -math.inf
        lp = (z - s["stats"][rows, :1].to(F64)) / tau - s["stats"][rows, 1:].to(F64)
        p = torch.exp(lp)
        hot = torch.zeros_like(p).scatter_(1, s["targets"][rows].to(I64)[:, None], 1.0)
        g = s["dlp"][rows, None].to(F64) * (hot - p)
        if s["dent"] is not None:
            tail = torch.where(p > 0, p * (lp + s["entropy"][rows, None].to(F64)), 0 * p)
            g -= s["dent"][rows, None].to(F64) * tail
        dead = (s["mask"][rows] == 0)[:, None] | (z == -math.inf) | \
            (s["stats"][rows, :1] == -math.inf)
        g[dead] = 0.0
        out[rows] = g / tau
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "logits":
        return _exact_logits(s)
    if op == "logits_grad":
        return {"grad": _exact_logits_grad(s)}
    if op == "head":
        z = s["hidden"][s["in_loss"]].to(F64) @ s["w"].to(F64).T / case["tau"]
        lse = torch.logsumexp(z, 1)
        lp = z.sub_(lse[:, None])
        y = s["targets"][s["in_loss"]].to(I64)[:, None]
        out = {}
        for name, v in (("logprob", lp.gather(1, y)[:, 0]), ("lse", lse),
                        ("entropy", -(torch.exp(lp) * lp).sum(1))):
            out[name] = torch.zeros(s["mask"].numel(), dtype=F64, device=DEV)
            out[name][s["in_loss"]] = v
        return out
    if op == "head_grad":
        dh, dw = _head_grad(s, F64)
        return {"grad_hidden": dh, "grad_w": dw}
    if op == "ortho":
        return {"update": _newton_schulz(s["x"].to(F64))}
    momentum, weight = _muon(case, s["x"], s["momentum"], s["weight"], F64)
    return {"momentum": momentum, "weight": weight, "weight_bf16": weight}
