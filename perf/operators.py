"""Operators of a mixture-of-experts layer around the token routing: cases, inputs, plain forms and exact values.

The layer is norm -> gate -> (routing) -> expert feed-forward over the rows grouped by slot -> (combine) -> dropout and
residual.  Four operators are measured, each with its backward pass where a training step has one:

  ffn      the experts' gated feed-forward block over the dispatched rows, grouped by destination slot
  norm     layer norm with the reduction of the gradients of its weight and bias
  gate     the K largest logits of a token, their normalised weights, and the gradient of the logits
  dropout  dropout from a counter-based generator, added to the residual stream

With `own` false `run` computes the plain form (elementary torch operations in 32 bits, rounded once at the end); with
`own` true it makes the calls of this repository's package.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ---- cases -------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of generation: six rows for six experts, their weights stream once through the chip
        dict(name="ffn one token, H 2048", op="ffn", T=1, K=6, E=64, spare=32, H=2048, F=1408, train=False),
        # a generation batch: a few rows for nearly every one of 128 experts, all their weights are read
        dict(name="ffn batch of 48, H 4096", op="ffn", T=48, K=8, E=128, spare=32, H=4096, F=1536, train=False),
        # a ragged prompt through many small experts: group ends inside tiles, F no multiple of the tile
        dict(name="ffn prompt 4999, H 2048", op="ffn", T=4999, K=6, E=64, spare=32, H=2048, F=1408, train=False),
        # a training step with few, large experts (top-2 of 8, replicated on 32 slots)
        dict(name="ffn train 8192, H 4096", op="ffn", T=8192, K=2, E=8, spare=24, H=4096, F=2816, train=True),
        # a training step at the width of the largest configuration, one GPU's share of experts
        dict(name="ffn train 8192, H 7168", op="ffn", T=8192, K=8, E=32, spare=4, H=7168, F=2048, train=True),
        # the norm in front of a layer, one token of generation
        dict(name="norm one token, H 7168", op="norm", T=1, H=7168, dtype="bf16", train=False),
        # the same norm in a training step over a whole batch
        dict(name="norm train 65536, H 7168", op="norm", T=65536, H=7168, dtype="bf16", train=True),
        # a 32-bit norm of odd sizes in training
        dict(name="norm train 4099, H 1000", op="norm", T=4099, H=1000, dtype="f32", train=True),
        # gating of a small batch in 16 bits, softmax over the chosen two of 16
        dict(name="gate 257 of 16", op="gate", T=257, E=16, K=2, kind="softmax", dtype="bf16", train=False),
        # gating of the largest configuration's step and its gradient, sigmoid renormalised over 8 of 256
        dict(name="gate train 131072 of 256", op="gate", T=131072, E=256, K=8, kind="sigmoid", dtype="f32", train=True),
        # dropout and residual of a short prompt in 32 bits, sizes that fill no whole block of threads
        dict(name="dropout 33 x 1000", op="dropout", T=33, H=1000, p=0.25, dtype="f32", train=False),
        # dropout and residual of a training step, both directions
        dict(name="dropout train 32768 x 7168", op="dropout", T=32768, H=7168, p=0.1, dtype="bf16", train=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["ffn", "ffn", "norm", "gate", "dropout"])
    train = rng.random() < 0.5
    if op == "ffn":
        while True:
            E, K = spread(4, 128), rng.randint(1, 8)
            c = dict(op=op, T=spread(1, 16384), K=min(K, E), E=E, spare=rng.randint(0, E), H=8 * spread(32, 896), F=8 * spread(16, 352), train=train)
            if c["T"] * c["K"] * c["H"] * c["F"] <= 65536 * 7168 * 2048 and E * c["H"] * c["F"] <= 128 * 4096 * 1536:
                return c
    if op == "norm":
        while True:
            c = dict(op=op, T=spread(1, 65536), H=8 * spread(1, 1024), dtype=rng.choice(["bf16", "f32"]), train=train)
            if c["T"] * c["H"] * (2 if c["dtype"] == "f32" else 1) <= 65536 * 7168:
                return c
    if op == "gate":
        while True:
            E = spread(4, 1024)
            c = dict(op=op, T=spread(1, 131072), E=E, K=rng.randint(1, min(16, E)), kind=rng.choice(["softmax", "sigmoid"]),
                     dtype=rng.choice(["bf16", "f32"]), train=train)
            if c["T"] * E <= 131072 * 256:
                return c
    while True:
        c = dict(op=op, T=spread(1, 65536), H=8 * spread(1, 1024), p=rng.choice([0.05, 0.1, 0.25, 0.5]), dtype=rng.choice(["bf16", "f32"]), train=train)
        if c["T"] * c["H"] * (2 if c["dtype"] == "f32" else 1) <= 32768 * 7168:
            return c


def work(case):
    c = case
    if c["op"] == "ffn":
        P, H, F = c["T"] * c["K"], c["H"], c["F"]
        used = c["E"] * (1.0 - (1.0 - c["K"] / c["E"]) ** c["T"])   # experts that some token reaches
        weights = 3 * 2.0 * used * H * F
        if not c["train"]:
            return {"bytes": weights + 2.0 * 2 * P * H, "flops": 6.0 * P * H * F}
        # rows and output gradient in, output and row gradient out; every expert's weight gradient is written
        return {"bytes": weights + 3 * 2.0 * c["E"] * H * F + 4 * 2.0 * P * H, "flops": 18.0 * P * H * F}
    if c["op"] == "gate":
        size = 4 if c["dtype"] == "f32" else 2
        n, k = float(c["T"]) * c["E"], float(c["T"]) * c["K"]
        return {"bytes": n * size + 8 * k + (n * size + 4 * k if c["train"] else 0), "flops": n + 6 * k + (6 * k if c["train"] else 0)}
    size, n = (4 if c["dtype"] == "f32" else 2), float(c["T"]) * c["H"]
    if c["op"] == "norm":
        # forward: x in, y out; a training step also reads the output's gradient and writes the input's
        return {"bytes": n * size * (4 if c["train"] else 2) + 8.0 * c["H"] * (2 if c["train"] else 1), "flops": n * (22 if c["train"] else 8)}
    return {"bytes": n * size * (5 if c["train"] else 3), "flops": n * (3 if c["train"] else 2)}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(shape, gen, dtype=torch.float32, scale=1.0, shift=0.0):
    t = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
    return t.mul_(scale).add_(shift) if shift else t.mul_(scale) if scale != 1.0 else t


def _ffn_inputs(case, seed):
    g = _gen(seed)
    T, K, E, H, F = (case[k] for k in ("T", "K", "E", "H", "F"))
    D = E + case["spare"]
    # every expert once, replicas of some in most of the spare slots, the last spare slot empty
    slot = torch.cat([torch.randperm(E, generator=g, device="cuda"), torch.randint(0, E, (case["spare"],), generator=g, device="cuda")])
    if case["spare"]:
        slot[-1] = -1
    # a token picks K distinct slots; slots differ in popularity as gating does
    popular = torch.log(1.0 / (1.0 + torch.randperm(D, generator=g, device="cuda").float()) ** 0.8)
    popular = torch.where(slot < 0, torch.full_like(popular, -math.inf), popular)
    noise = -torch.log(-torch.log(torch.rand((T, D), generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)))
    counts = torch.bincount((popular + noise).topk(K, dim=1).indices.reshape(-1), minlength=D)
    offsets = torch.zeros(D + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = counts.cumsum(0)
    host, experts = offsets.tolist(), slot.tolist()
    ranges = {}
    for d, e in enumerate(experts):
        if e >= 0 and host[d + 1] > host[d]:
            ranges.setdefault(e, []).append((host[d], host[d + 1]))
    s = {"rows": _randn((T * K, H), g, torch.bfloat16),
         "w_gate_up": _randn((E, 2 * F, H), g, torch.bfloat16, H ** -0.5),
         "w_down": _randn((E, H, F), g, torch.bfloat16, F ** -0.5),
         "dest_offsets": offsets.to(torch.int32), "slot_expert": slot.to(torch.int32), "ranges": sorted(ranges.items())}
    if case["train"]:
        s["grad_out"] = _randn((T * K, H), g, torch.bfloat16)
    return s


def _norm_inputs(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    T, H = case["T"], case["H"]
    s = {"x": _randn((T, H), g, dt, 2.0, 0.5), "gamma": _randn((H,), g, scale=0.2, shift=1.0), "beta": _randn((H,), g, scale=0.1)}
    if case["train"]:
        s["grad_y"] = _randn((T, H), g, dt)
    return s


def _gate_inputs(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    s = {"logits": _randn((case["T"], case["E"]), g, dt), "K": case["K"], "kind": case["kind"]}
    if case["train"]:
        s["grad_w"] = _randn((case["T"], case["K"]), g)
    return s


def _dropout_inputs(case, seed):
    g, dt = _gen(seed), DTYPES[case["dtype"]]
    shape = (case["T"], case["H"])
    s = {"x": _randn(shape, g, dt), "residual": _randn(shape, g, dt), "p": case["p"], "seed": (int(seed) * 0x9E3779B97F4A7C15 + 1) % 2**64}
    if case["train"]:
        s["grad_out"] = _randn(shape, g, dt)
    return s


INPUTS = {"ffn": _ffn_inputs, "norm": _norm_inputs, "gate": _gate_inputs, "dropout": _dropout_inputs}


def prepare(case, seed):
    s = INPUTS[case["op"]](case, seed)
    s["op"], s["train"] = case["op"], case["train"]
    if own:
        s["buffers"] = _buffers(s)   # outputs and workspace, which a program allocates once and passes to every call
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _ffn_plain(s):
    F = s["w_down"].shape[2]
    out = torch.zeros_like(s["rows"])
    if s["train"]:
        grad_rows = torch.zeros_like(s["rows"])
        grad_gate_up, grad_down = torch.zeros_like(s["w_gate_up"]), torch.zeros_like(s["w_down"])
    for e, ranges in s["ranges"]:      # the grouped product: one dense block for each expert that has rows
        x = torch.cat([s["rows"][a:b] for a, b in ranges]).float()
        sizes = [b - a for a, b in ranges]
        w_gate_up, w_down = s["w_gate_up"][e].float(), s["w_down"][e].float()
        pre = x @ w_gate_up.t()
        gate, up = pre[:, :F], pre[:, F:]
        sig = 1.0 / (1.0 + torch.exp(-gate))
        act = gate * sig * up
        y = act @ w_down.t()
        for (a, b), part in zip(ranges, y.split(sizes)):
            out[a:b] = part.to(out.dtype)
        if s["train"]:
            dy = torch.cat([s["grad_out"][a:b] for a, b in ranges]).float()
            d_act = dy @ w_down
            d_pre = torch.cat([d_act * up * sig * (1.0 + gate * (1.0 - sig)), d_act * gate * sig], dim=1)
            grad_down[e] = (dy.t() @ act).to(grad_down.dtype)
            grad_gate_up[e] = (d_pre.t() @ x).to(grad_gate_up.dtype)
            for (a, b), part in zip(ranges, (d_pre @ w_gate_up).split(sizes)):
                grad_rows[a:b] = part.to(grad_rows.dtype)
    return (out, grad_rows, grad_gate_up, grad_down) if s["train"] else out


def _norm_plain(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    xhat = centred * rstd
    y = (xhat * s["gamma"] + s["beta"]).to(s["x"].dtype)
    if not s["train"]:
        return y
    dy = s["grad_y"].float()
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return y, dx.to(s["x"].dtype), (dy * xhat).sum(dim=0), dy.sum(dim=0)


def _gate_plain(s):
    logits = s["logits"].float()
    value, ids = torch.sort(logits, dim=1, descending=True, stable=True)   # stable: ties go to the lowest id
    value, ids = value[:, :s["K"]], ids[:, :s["K"]]
    if s["kind"] == "softmax":
        score = torch.exp(value - value[:, :1])
    else:
        score = 1.0 / (1.0 + torch.exp(-value))
    w = score / score.sum(dim=1, keepdim=True)
    if not s["train"]:
        return ids.to(torch.int32), w
    dl = w * (s["grad_w"] - (s["grad_w"] * w).sum(dim=1, keepdim=True))
    if s["kind"] == "sigmoid":
        dl = dl * (1.0 - score)
    grad = torch.zeros_like(logits).scatter_(1, ids, dl)
    return ids.to(torch.int32), w, grad.to(s["logits"].dtype)


def _philox(blocks, seed):
    """Philox-4x32-10 (Salmon et al., SC 2011) of the counters (block, 0) under the key `seed`: [blocks, 4] words."""
    low = 0xFFFFFFFF
    b = torch.arange(blocks, device="cuda", dtype=torch.int64)
    c0, c1 = b & low, b >> 32
    c2, c3 = torch.zeros_like(b), torch.zeros_like(b)
    k0, k1 = seed & low, seed >> 32

    def high(c, m):   # the upper 32 bits of a 64-bit product, without leaving int64
        return (c * (m >> 16) + ((c * (m & 0xFFFF)) >> 16)) >> 16

    for _ in range(10):
        c0, c1, c2, c3 = (high(c2, 0xCD9E8D57) ^ c1 ^ k0, (c2 * 0xCD9E8D57) & low,
                          high(c0, 0xD2511F53) ^ c3 ^ k1, (c0 * 0xD2511F53) & low)
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], dim=1)


def _keep(shape, p, seed):
    """Element i is kept where half-word i % 8 of block i / 8 is at least the threshold."""
    n = shape[0] * shape[1]
    words = _philox((n + 7) // 8, seed)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)[:n]
    return (halves >= _threshold(p)).reshape(shape)


def _threshold(p):
    return min(65535, int(p * 65536.0 + 0.5))


def _dropout_plain(s):
    keep = _keep(s["x"].shape, s["p"], s["seed"])
    scale = 65536.0 / (65536 - _threshold(s["p"]))
    zero = torch.zeros((), device="cuda")
    out = (s["residual"].float() + torch.where(keep, s["x"].float() * scale, zero)).to(s["x"].dtype)
    if not s["train"]:
        return out
    return out, torch.where(keep, s["grad_out"].float() * scale, zero).to(s["x"].dtype)


PLAIN = {"ffn": _ffn_plain, "norm": _norm_plain, "gate": _gate_plain, "dropout": _dropout_plain}


# ---- this repository's calls -------------------------------------------------------------------------------------

def _buffers(s):
    import paper_2609_36959_b200 as cb

    def like(t):
        return torch.empty_like(t)

    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if s["op"] == "ffn":
        (P, H), (E, _, F), D = s["rows"].shape, s["w_down"].shape, s["slot_expert"].numel()
        b = {"out": like(s["rows"]), "act": new(P, F, dtype=torch.bfloat16), "pre": None,
             "workspace": new(cb.expert_ffn_workspace_bytes(P, D, E, H, F), dtype=torch.uint8)}
        if s["train"]:
            b.update(pre=new(P, 2 * F, dtype=torch.bfloat16), grad_pre=new(P, 2 * F, dtype=torch.bfloat16), grad_rows=like(s["rows"]),
                     grad_w_gate_up=like(s["w_gate_up"]), grad_w_down=like(s["w_down"]))
        return b
    if s["op"] == "norm":
        T, H = s["x"].shape
        b = {"y": like(s["x"]), "mean": new(T), "rstd": new(T)}
        if s["train"]:
            b.update(grad_x=like(s["x"]), grad_gamma=new(H), grad_beta=new(H), workspace=new(cb.layer_norm_workspace_bytes(T, H), dtype=torch.uint8))
        return b
    if s["op"] == "gate":
        T = s["logits"].shape[0]
        b = {"ids": new(T, s["K"], dtype=torch.int32), "w": new(T, s["K"]), "flags": cb.GATE_SIGMOID if s["kind"] == "sigmoid" else 0}
        if s["train"]:
            b["grad_logits"] = like(s["logits"])
        return b
    return {"out": like(s["x"]), "grad_x": like(s["x"]) if s["train"] else None}


def _ffn_own(s, b, cb):
    cb.expert_ffn(s["rows"], s["dest_offsets"], s["slot_expert"], s["w_gate_up"], s["w_down"], b["act"], b["out"], b["workspace"], pre=b["pre"])
    if not s["train"]:
        return b["out"]
    cb.expert_ffn_backward(s["grad_out"], s["rows"], s["dest_offsets"], s["slot_expert"], s["w_gate_up"], s["w_down"], b["pre"], b["act"],
                           b["grad_pre"], b["workspace"], grad_rows=b["grad_rows"], grad_w_gate_up=b["grad_w_gate_up"], grad_w_down=b["grad_w_down"])
    return b["out"], b["grad_rows"], b["grad_w_gate_up"], b["grad_w_down"]


def _norm_own(s, b, cb):
    cb.layer_norm(s["x"], s["gamma"], s["beta"], EPS, b["y"], b["mean"], b["rstd"])
    if not s["train"]:
        return b["y"]
    cb.layer_norm_backward(s["grad_y"], s["x"], s["gamma"], b["mean"], b["rstd"], b["grad_x"], b["grad_gamma"], b["grad_beta"], b["workspace"])
    return b["y"], b["grad_x"], b["grad_gamma"], b["grad_beta"]


def _gate_own(s, b, cb):
    cb.gate_topk(s["logits"], b["ids"], b["w"], flags=b["flags"])
    if not s["train"]:
        return b["ids"], b["w"]
    cb.gate_topk_backward(s["grad_w"], s["logits"], b["ids"], b["w"], b["grad_logits"], flags=b["flags"])
    return b["ids"], b["w"], b["grad_logits"]


def _dropout_own(s, b, cb):
    cb.dropout_add(s["x"], s["residual"], s["p"], s["seed"], b["out"])
    if not s["train"]:
        return b["out"]
    cb.dropout_add_backward(s["grad_out"], s["p"], s["seed"], b["grad_x"])
    return b["out"], b["grad_x"]


OWN = {"ffn": _ffn_own, "norm": _norm_own, "gate": _gate_own, "dropout": _dropout_own}


def run(state):
    if not own:
        return PLAIN[state["op"]](state)
    import paper_2609_36959_b200 as cb
    return OWN[state["op"]](state, state["buffers"], cb)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _ffn_exact(s):
    F = s["w_down"].shape[2]
    P, H = s["rows"].shape
    out, dx = (torch.zeros((P, H), dtype=torch.float64, device="cuda") for _ in range(2))
    d_gu = torch.zeros(s["w_gate_up"].shape, dtype=torch.float64, device="cuda") if s["train"] else None
    d_dn = torch.zeros(s["w_down"].shape, dtype=torch.float64, device="cuda") if s["train"] else None
    for e, ranges in s["ranges"]:
        wg, wu = s["w_gate_up"][e, :F].double(), s["w_gate_up"][e, F:].double()
        wd = s["w_down"][e].double()
        for a, b in ranges:            # slot by slot; an expert's weight gradients add up over its replicas
            x = s["rows"][a:b].double()
            g, u = torch.einsum("mh,fh->mf", x, wg), torch.einsum("mh,fh->mf", x, wu)
            silu = g * torch.special.expit(g)
            out[a:b] = torch.einsum("mf,hf->mh", silu * u, wd)
            if s["train"]:
                dy = s["grad_out"][a:b].double()
                da = torch.einsum("mh,hf->mf", dy, wd)
                q = torch.special.expit(g)
                dg, du = da * u * (q + silu * (1 - q)), da * silu
                dx[a:b] = torch.einsum("mf,fh->mh", dg, wg) + torch.einsum("mf,fh->mh", du, wu)
                d_gu[e, :F] += torch.einsum("mf,mh->fh", dg, x)
                d_gu[e, F:] += torch.einsum("mf,mh->fh", du, x)
                d_dn[e] += torch.einsum("mh,mf->hf", dy, silu * u)
    return (out, dx, d_gu, d_dn) if s["train"] else out


def _norm_exact(s):
    x = s["x"].double()
    var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    sigma = (var + EPS).sqrt()
    z = (x - mu) / sigma
    y = z * s["gamma"].double() + s["beta"].double()
    if not s["train"]:
        return y
    dy = s["grad_y"].double()
    dz = dy * s["gamma"].double()
    H = x.shape[1]
    dx = (H * dz - dz.sum(1, keepdim=True) - z * (dz * z).sum(1, keepdim=True)) / (H * sigma)
    return y, dx, torch.einsum("th,th->h", dy, z), dy.sum(0)


def _gate_exact(s):
    logits = s["logits"].double()
    T, E = logits.shape
    left = logits.clone()
    ids = torch.empty((T, s["K"]), dtype=torch.int64, device="cuda")
    column = torch.arange(E, device="cuda").expand(T, E)
    for k in range(s["K"]):            # the largest that is left, at its lowest place
        at = torch.where(left == left.amax(1, keepdim=True), column, E).amin(1)
        ids[:, k] = at
        left.scatter_(1, at[:, None], -math.inf)
    v = logits.gather(1, ids)
    w = torch.softmax(v, 1) if s["kind"] == "softmax" else torch.sigmoid(v) / torch.sigmoid(v).sum(1, keepdim=True)
    if not s["train"]:
        return ids.to(torch.int32), w
    g = s["grad_w"].double()
    if s["kind"] == "softmax":
        d = w * g - w * (w * g).sum(1, keepdim=True)
    else:
        q = torch.sigmoid(v)
        total = q.sum(1, keepdim=True)
        d = q * (1 - q) * (g / total - (g * q).sum(1, keepdim=True) / total ** 2)
    return ids.to(torch.int32), w, torch.zeros_like(logits).scatter_add_(1, ids, d)


def _dropout_exact(s):
    t = _threshold(s["p"])
    kept = _keep(s["x"].shape, s["p"], s["seed"]).double() * (65536.0 / (65536 - t))
    out = s["residual"].double() + kept * s["x"].double()
    return (out, kept * s["grad_out"].double()) if s["train"] else out


EXACT = {"ffn": _ffn_exact, "norm": _norm_exact, "gate": _gate_exact, "dropout": _dropout_exact}


def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    s["op"], s["train"] = case["op"], case["train"]
    return EXACT[case["op"]](s)
