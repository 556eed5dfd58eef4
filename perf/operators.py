"""Timed cases of the router's training operators and of the 8-bit expert products.

Each case names an operation ("op"):
  quantize  fp8_quantize: e4m3 values with a float32 scale for every 128 columns of a row, or for
            every 128 x 128 block of a matrix
  matmul    fp8_matmul: row segments of an 8-bit matrix by each group's 8-bit weights
  moe       fp8_moe_forward: routed tokens through 8-bit expert networks, combined
  balance   balance_loss: per-expert counts, the load balance loss and its gradient
  gate_bwd  group_gate_backward: gradients of the two-stage group gate

Shapes are those of the package's own workloads, and generic ragged ones. Inputs follow the
distributions of those workloads: hidden states of unit root mean square, normal weights, expert
popularity uniform or Zipf. With `own` false run() is the operators' plain form in float32; exact()
is their definition in float64.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 128        # values that share a scale
FP8_MAX = 448.0    # the largest e4m3 value
AMAX_MIN = 2.0 ** -100  # a block of smaller values is scaled as if this were its largest


def listed():
    return [
        # the hidden states of one decoding step (32 sequences, one token each): latency counts
        dict(name="quantize_decode", op="quantize", dtype="bf16", mats=1, rows=32, cols=4096, block_rows=1),
        # the expert weights of a layer, prepared once when it is loaded
        dict(name="quantize_weights", op="quantize", dtype="bf16", mats=64, rows=2816, cols=2048, block_rows=128),
        # one token by one weight matrix: a stream of the weights
        dict(name="matmul_token", op="matmul", rows=1, G=1, n=4096, k=4096, out="bf16", tail=0),
        # ragged segments of a prefill batch, one of them empty, an odd width, rows behind the last segment
        dict(name="matmul_segments", op="matmul", rows=3000, G=12, n=2001, k=2048, out="f32", tail=37),
        # one decoding step through 64 experts
        dict(name="moe_decode", op="moe", T=32, d=4096, M=64, H=1536, k=8, keep=40, zipf=0.0, act="swiglu"),
        # prefill over many small experts of unequal popularity
        dict(name="moe_finegrained", op="moe", T=8192, d=2048, M=64, H=1408, k=6, keep=48, zipf=1.1, act="swiglu"),
        # prefill through 8 large experts
        dict(name="moe_mixtral", op="moe", T=4096, d=4096, M=8, H=14336, k=2, keep=8, zipf=0.0, act="swiglu"),
        # the router's loss on a batch, and on a long one with padded sequences
        dict(name="balance_finegrained", op="balance", T=8192, M=64, K=8, k=6, keep=48, pad=0.0),
        dict(name="balance_long", op="balance", T=131129, M=256, K=16, k=8, keep=256, pad=0.2),
        # the router's gradients: the smallest layer in float32, a batch over many small experts,
        # a wide batch with few experts
        dict(name="gate_bwd_tiny_f32", op="gate_bwd", dtype="f32", T=64, d=128, M=8, K=2, k=2, keep=6, uneven=False,
             renorm=True, pad=0.0, full=False),
        dict(name="gate_bwd_finegrained", op="gate_bwd", dtype="bf16", T=8192, d=2048, M=64, K=8, k=6, keep=48,
             uneven=False, renorm=True, pad=0.0, full=False),
        dict(name="gate_bwd_mixtral", op="gate_bwd", dtype="bf16", T=4096, d=4096, M=8, K=2, k=2, keep=8, uneven=False,
             renorm=True, pad=0.1, full=True),
    ]


# ----------------------------------------------------------------------------- more of the same

MAX_FLOPS = 2.8e12          # below the largest listed case
MAX_WEIGHTS = 1.4e9         # 8-bit weights of a case
MAX_PADDED = 6e9            # values of the plain form's padded batches


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    return BLOCK * _log_int(rng, lo // BLOCK, hi // BLOCK)


def _routing(rng):
    M = rng.choice((8, 16, 32, 64, 128))
    keep = rng.randint(max(2, M // 4), M)
    return M, keep, rng.randint(1, min(8, keep))


def _groups(M):
    K = 1
    while (2 * K) * (2 * K) <= M:
        K *= 2
    return K


def _draw(rng):
    op = rng.choices(("quantize", "matmul", "moe", "balance", "gate_bwd"), (2, 3, 4, 2, 3))[0]
    if op == "quantize":
        mats = rng.choice((1, 1, 1, 4, 16))
        return dict(op=op, dtype=rng.choice(("bf16", "bf16", "f32")), mats=mats, rows=_log_int(rng, 1, 16384 // mats),
                    cols=_width(rng, 128, 8192), block_rows=rng.choice((1, 1, 128)))
    if op == "matmul":
        G = rng.choice((1, 1, 4, 16, 64))
        rows = _log_int(rng, 1, 16384)
        return dict(op=op, rows=rows, G=G, n=_log_int(rng, 16, 8192), k=_width(rng, 128, 8192),
                    out=rng.choice(("bf16", "bf16", "f32")), tail=rng.choice((0, 0, rng.randint(1, 40))) if G > 1 else 0)
    if op == "moe":
        M, keep, k = _routing(rng)
        return dict(op=op, T=_log_int(rng, 1, 8192), d=_width(rng, 512, 4096), M=M, H=_width(rng, 512, 8192), k=k,
                    keep=keep, zipf=rng.choice((0.0, 0.0, 1.1)), act=rng.choice(("swiglu", "swiglu", "relu")))
    M, keep, k = _routing(rng)
    if op == "balance":
        return dict(op=op, T=_log_int(rng, 1, 131072), M=M, K=_groups(M), k=k, keep=keep, pad=rng.choice((0.0, 0.3)))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    # a single selected weight that is renormalised is 1 whatever the router says: nothing to measure
    return dict(op=op, dtype=dtype, T=_log_int(rng, 2, 8192), d=_width(rng, 128, 4096), M=M, K=_groups(M),
                k=max(2, k), keep=max(keep, 4), uneven=rng.random() < 0.3, renorm=rng.random() < 0.7,
                pad=rng.choice((0.0, 0.3)), full=rng.random() < 0.5)


def _fits(case):
    op = case["op"]
    if op == "matmul":
        if case["G"] * case["n"] * case["k"] > MAX_WEIGHTS:
            return False
        if case["G"] * case["rows"] * max(case["n"], case["k"]) > MAX_PADDED:
            return False
    if op == "moe":
        if case["M"] * (_w_in_rows(case) + case["H"]) * case["d"] > MAX_WEIGHTS:
            return False
        if case["M"] * case["T"] * (_w_in_rows(case) + case["d"]) > MAX_PADDED:
            return False
    return work(case)["flops"] <= MAX_FLOPS


def draw(rng):
    while True:
        case = _draw(rng)
        if _fits(case):
            return case


# ----------------------------------------------------------------------------- inputs

def _w_in_rows(case):
    return case["H"] if case["act"] == "relu" else 2 * case["H"]


def _group_sizes(case):
    """Equal groups of experts, or every second group giving half its experts to its neighbour."""
    M, K = case["M"], case["K"]
    sizes = [M // K] * K
    if case.get("uneven"):
        for i in range(0, K - 1, 2):
            move = sizes[i] // 2
            sizes[i] -= move
            sizes[i + 1] += move
    return sizes


class _Draw:
    def __init__(self, seed):
        self.gpu = torch.Generator(device=DEV)
        self.gpu.manual_seed(seed)
        self.cpu = torch.Generator()
        self.cpu.manual_seed(seed)

    def normal(self, shape, std, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=self.gpu)

    def hidden(self, rows, d, dtype=torch.float32):
        """Hidden states with rows of unit root mean square, a few channels ten times the others."""
        x = self.normal((rows, d), 1.0)
        x[:, torch.randperm(d, generator=self.cpu)[: d // 64].to(DEV)] *= 10.0
        return (x * torch.rsqrt(x.square().mean(dim=1, keepdim=True))).to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.gpu, device=DEV)

    def scores(self, T, M, keep, zipf):
        """Scores whose largest are the routed experts: distinct candidates by popularity."""
        s = -torch.log(-torch.log(self.uniform((T, M)).clamp_(1e-7, 1 - 1e-7)))
        order = torch.randperm(M, generator=self.cpu)
        if zipf:
            s += (-zipf * (order + 1).double().log()).float().to(DEV)
        s[:, torch.randperm(M, generator=self.cpu)[keep:].to(DEV)] = -math.inf
        return s

    def weights8(self, mats, rows, cols):
        """8-bit weights with a scale per block, one matrix at a time."""
        q = torch.empty((mats, rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
        s = torch.empty((mats, -(-rows // BLOCK), cols // BLOCK), dtype=torch.float32, device=DEV)
        for i in range(mats):
            qi, si = _quantize(self.normal((1, rows, cols), 0.02), BLOCK)
            q[i], s[i] = qi[0], si[0]
        return q, s


def _segments(case, g):
    """G + 1 offsets of ragged segments (every fifth empty) over all rows but the tail."""
    G, rows = case["G"], case["rows"] - min(case["tail"], case["rows"] - 1)
    share = torch.rand(G, generator=g.cpu).double() + 0.05
    share[4::5] = 0.0
    seg = torch.round(torch.cumsum(share / share.sum(), 0) * rows).to(torch.int32)
    return torch.cat([torch.zeros(1, dtype=torch.int32), seg])


def prepare(case, seed):
    g = _Draw(seed)
    op = case["op"]
    s = {"op": op, "case": case}
    if op == "quantize":
        dt = DTYPES[case["dtype"]]
        if case["block_rows"] == 1:
            s["x"] = g.hidden(case["mats"] * case["rows"], case["cols"], dt).reshape(case["mats"], case["rows"], case["cols"])
        else:
            s["x"] = g.normal((case["mats"], case["rows"], case["cols"]), 0.02, dt)
    elif op == "matmul":
        s["a"], s["a_scale"] = (t[0] for t in _quantize(g.hidden(case["rows"], case["k"])[None], 1))
        s["b"], s["b_scale"] = g.weights8(case["G"], case["n"], case["k"])
        s["seg"] = _segments(case, g).to(DEV) if case["G"] > 1 else None
        # rows behind the last segment belong to the caller and stay as they are
        s["out"] = torch.zeros((case["rows"], case["n"]), dtype=DTYPES[case["out"]], device=DEV)
    elif op == "moe":
        s["x"] = g.hidden(case["T"], case["d"], torch.bfloat16)
        val, idx = torch.topk(g.scores(case["T"], case["M"], case["keep"], case["zipf"]), case["k"], dim=1)
        s["idx"], s["w"] = idx.to(torch.int32).contiguous(), torch.softmax(val, dim=1).contiguous()
        s["w_in"], s["w_in_scale"] = g.weights8(case["M"], _w_in_rows(case), case["d"])
        s["w_down"], s["w_down_scale"] = g.weights8(case["M"], case["d"], case["H"])
    else:
        T, M, K, k = case["T"], case["M"], case["K"], case["k"]
        sizes = _group_sizes(case)
        off = torch.randperm(M, generator=g.cpu)[case["keep"]:].to(DEV)
        group = torch.repeat_interleave(torch.arange(K), torch.tensor(sizes)).to(DEV)
        if op == "gate_bwd":
            dt = DTYPES[case["dtype"]]
            s["x"] = g.hidden(T, case["d"], dt)
            s["w_global"], s["w_local"] = (g.normal((n, case["d"]), 0.02, dt) for n in (K, M))
            local = s["x"].double() @ s["w_local"].double().t()
            glob = s["x"].double() @ s["w_global"].double().t()
        else:
            local, glob = g.normal((T, M), 1.5).double(), g.normal((T, K), 1.0).double()
        s["probs"] = _gate_probs(local, glob, off, group, K).float().contiguous()
        s["idx"] = torch.sort(s["probs"], dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32).contiguous()
        s["valid"] = (g.uniform((T,)) >= case["pad"]) if case["pad"] else None
        s["sizes"], s["group"], s["K"], s["k"] = sizes, group, K, k
        if op == "gate_bwd":
            s["d_topk_w"] = g.normal((T, k), 1.0)
            s["d_probs"] = g.normal((T, M), 0.1) if case["full"] else None
            s["d_balance"] = g.uniform((M,)) * 0.02
            s["renorm"] = case["renorm"]
    return s


def _gate_probs(local, glob, off, group, K):
    """The gate's distribution: softmax over the groups that hold a candidate times the softmax
    over each group's candidates."""
    local = local.clone()
    local[:, off] = -math.inf
    # scatter each expert's logit to its group's slots: [T][K][M], -inf elsewhere
    member = torch.nn.functional.one_hot(group, K).t().bool()
    live = torch.isfinite(local[0]) & member
    glob = glob.masked_fill(~live.any(dim=1), -math.inf)
    pg = torch.softmax(glob, dim=1)
    top = torch.stack([local.masked_fill(~live[i], -math.inf).amax(dim=1) for i in range(K)], dim=1)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    e = torch.exp(local - top[:, group])
    z = e @ member.t().double()
    return e / torch.where(z > 0, z, torch.ones_like(z))[:, group] * pg[:, group]


# ----------------------------------------------------------------------------- the plain forms

def _quantize(x, block_rows):
    """x [mats][rows][cols] -> (e4m3 values, float32 scales): per block of block_rows x 128 the
    largest value maps to 448."""
    mats, rows, cols = x.shape
    nb = -(-rows // block_rows)
    f = x.float()
    if nb * block_rows != rows:
        f = torch.nn.functional.pad(f, (0, 0, 0, nb * block_rows - rows))
    f = f.reshape(mats, nb, block_rows, cols // BLOCK, BLOCK)
    amax = f.abs().amax(dim=(2, 4)).clamp_min(AMAX_MIN)
    # a tensor by a tensor: torch multiplies by the reciprocal when the divisor is a number. The
    # quotient 448 x / amax is rounded once, so that bfloat16 values half way between two e4m3
    # values (about one in a thousand) are seen as such
    scale = amax / torch.full_like(amax, FP8_MAX)
    q = (f * FP8_MAX / amax[:, :, None, :, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
    return q.reshape(mats, nb * block_rows, cols)[:, :rows].contiguous(), scale


def _values(q, scale, block_rows):
    """The float32 values that 8-bit numbers and their scales stand for; [rows][cols] or
    [mats][rows][cols]."""
    rows = q.shape[-2]
    s = scale.repeat_interleave(block_rows, dim=-2)[..., :rows, :]
    return (q.float().unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _slots(group, G):
    """Place of every row within its group (rows in any order) and the longest group's length."""
    order = torch.sort(group, stable=True).indices
    count = (group[:, None] == torch.arange(G, device=group.device)).sum(dim=0)
    first = torch.cumsum(count, 0) - count
    place = torch.empty_like(order)
    place[order] = torch.arange(group.numel(), device=group.device) - first[group[order]]
    return place, max(1, int(count.max()))


def _batched(rows, group, place, cap, w):
    """rows[i] @ w[group[i]].T as one batched float32 product over groups padded to cap rows."""
    pad = torch.zeros((w.shape[0], cap, rows.shape[1]), device=rows.device)
    pad[group, place] = rows
    return torch.bmm(pad, w.transpose(1, 2))


def _plain_matmul(s):
    a = _values(s["a"], s["a_scale"], 1)
    w = _values(s["b"], s["b_scale"], BLOCK)
    out = s["out"]
    if s["seg"] is None:
        out.copy_(a @ w[0].t())
        return {"out": out}
    at = torch.arange(a.shape[0], device=DEV)
    group = torch.searchsorted(s["seg"][1:].long(), at, right=True)
    held = torch.nonzero(group < w.shape[0]).flatten()
    group = group[held]
    place, cap = _slots(group, w.shape[0])
    out[held] = _batched(a[held], group, place, cap, w)[group, place].to(out.dtype)
    return {"out": out}


def _plain_moe(s):
    T, k = s["idx"].shape
    H = s["w_down"].shape[2]
    x = _values(*(t[0] for t in _quantize(s["x"][None], 1)), 1)
    group = s["idx"].reshape(-1).long()
    place, cap = _slots(group, s["w_down"].shape[0])
    h = _batched(x.repeat_interleave(k, dim=0), group, place, cap, _values(s["w_in"], s["w_in_scale"], BLOCK))
    if s["case"]["act"] == "relu":
        h = h.clamp_min(0.0)
    else:
        gate, up = h[..., :H], h[..., H:]
        h = gate / (1.0 + torch.exp(-gate)) * up
    h = _values(*_quantize(h, 1), 1)
    y = torch.bmm(h, _values(s["w_down"], s["w_down_scale"], BLOCK).transpose(1, 2))[group, place]
    return {"y": (y.reshape(T, k, -1) * s["w"].unsqueeze(2)).sum(dim=1).to(torch.bfloat16)}


def _plain_balance(s):
    probs, idx, M = s["probs"], s["idx"], s["case"]["M"]
    T, k = idx.shape
    valid = torch.ones(T, dtype=torch.bool, device=DEV) if s["valid"] is None else s["valid"]
    n = valid.sum().clamp_min(1).double()
    hit = (idx[:, :, None] == torch.arange(M, device=DEV)).sum(dim=1) * valid[:, None]
    counts = hit.sum(dim=0)
    d_probs = COEF * M * counts.double() / (k * n * n)
    loss = (d_probs * (probs.double() * valid[:, None]).sum(dim=0)).sum()
    return {"loss": loss.float().reshape(1), "counts": counts.to(torch.int32), "d_probs": d_probs.float()}


def _gate_grad(s, real):
    """Gradients of the gate's logits [T][M + K] in the type `real`, from its probabilities."""
    g, idx = s["probs"].to(real), s["idx"].long()
    T, M = g.shape
    valid = torch.ones(T, device=DEV, dtype=real) if s["valid"] is None else s["valid"].to(real)
    dw = s["d_topk_w"].to(real)
    if s["renorm"]:
        sel = torch.gather(g, 1, idx)
        total = sel.sum(dim=1, keepdim=True)
        w = sel / total
        dw = (dw - (w * dw).sum(dim=1, keepdim=True)) / total
    dg = s["d_balance"].to(real).expand(T, M).clone()
    if s["d_probs"] is not None:
        dg += s["d_probs"].to(real)
    dg.scatter_add_(1, idx, dw)
    member = torch.nn.functional.one_hot(s["group"], s["K"]).to(real)
    gd = g * dg * valid[:, None]
    a, p = gd @ member, g @ member
    share = g / torch.where(p > 0, p, torch.ones_like(p))[:, s["group"]]
    local = gd - share * a[:, s["group"]]
    glob = a - p * a.sum(dim=1, keepdim=True)
    return local, glob


def _gate_bwd(s, real):
    local, glob = _gate_grad(s, real)
    x, wl, wg = (s[n].to(real) for n in ("x", "w_local", "w_global"))
    out = torch.float64 if real == torch.float64 else torch.float32
    return {"d_x": (local @ wl + glob @ wg).to(s["x"].dtype if real == torch.float32 else out),
            "d_w_global": glob.t() @ x, "d_b_global": glob.double().sum(dim=0).to(out),
            "d_w_local": local.t() @ x, "d_b_local": local.double().sum(dim=0).to(out)}


COEF = 0.01  # the loss's usual weight beside the task's


def _plain(s):
    op = s["op"]
    if op == "quantize":
        q, scale = _quantize(s["x"], s["case"]["block_rows"])
        return {"q": q, "scale": scale}
    if op == "matmul":
        return _plain_matmul(s)
    if op == "moe":
        return _plain_moe(s)
    if op == "balance":
        return _plain_balance(s)
    return _gate_bwd(s, torch.float32)


# ----------------------------------------------------------------------------- the calls

def _calls(s):
    """What a program keeps from step to step: descriptors, outputs and workspaces."""
    from paper_2508_06024_amd import ec2moe as E
    c, op = s["case"], s["op"]
    new = lambda shape, dt: torch.empty(shape, dtype=dt, device=DEV)
    if op == "quantize":
        shape = (c["mats"], c["rows"], c["cols"])
        q = new(shape, torch.float8_e4m3fn)
        scale = new((c["mats"], -(-c["rows"] // c["block_rows"]), c["cols"] // BLOCK), torch.float32)
        return lambda: (E.fp8_quantize_into(s["x"], q, scale, c["block_rows"]), {"q": q, "scale": scale})[1]
    if op == "matmul":
        desc = E.fp8_matmul_desc(c["rows"], c["G"], c["n"], c["k"], DTYPES[c["out"]])
        ws = E.workspace(E.fp8_matmul_workspace_size(desc), DEV)
        return lambda: (E.fp8_matmul_into(desc, s["a"], s["a_scale"], s["seg"], s["b"], s["b_scale"], s["out"], ws),
                        {"out": s["out"]})[1]
    if op == "moe":
        desc = E.moe_desc(c["T"], c["M"], 1, c["d"], c["H"], c["k"], torch.bfloat16, activation=c["act"])
        ws = E.workspace(E.fp8_moe_workspace_size(desc), DEV)
        y = new((c["T"], c["d"]), torch.bfloat16)
        return lambda: (E.fp8_moe_forward_into(desc, s["x"], s["idx"], s["w"], s["w_in"], s["w_in_scale"], s["w_down"],
                                               s["w_down_scale"], y, ws), {"y": y})[1]
    if op == "balance":
        desc = E.moe_desc(c["T"], c["M"], c["K"], 128, 128, c["k"], torch.bfloat16)
        ws = E.workspace(E.balance_loss_workspace_size(desc), DEV)
        loss, counts, d_probs = new((1,), torch.float32), new((c["M"],), torch.int32), new((c["M"],), torch.float32)
        return lambda: (E.balance_loss_into(desc, s["probs"], s["idx"], COEF, loss, counts, d_probs, ws,
                                            token_valid=s["valid"]),
                        {"loss": loss, "counts": counts, "d_probs": d_probs})[1]
    desc = E.moe_desc(c["T"], c["M"], c["K"], c["d"], 128, c["k"], DTYPES[c["dtype"]], renormalize=c["renorm"])
    opts = E.gate_opts(0, s["sizes"] if c["uneven"] else None)
    ws = E.workspace(E.gate_backward_workspace_size(desc), DEV)
    out = {"d_x": torch.empty_like(s["x"]), "d_w_global": new((c["K"], c["d"]), torch.float32),
           "d_b_global": new((c["K"],), torch.float32), "d_w_local": new((c["M"], c["d"]), torch.float32),
           "d_b_local": new((c["M"],), torch.float32)}
    return lambda: (E.group_gate_backward_into(desc, opts, s["x"], s["w_global"], s["w_local"], s["probs"], s["idx"], ws,
                                               d_topk_w=s["d_topk_w"], d_probs=s["d_probs"], d_balance=s["d_balance"],
                                               token_valid=s["valid"], **out), out)[1]


def run(s):
    if own:
        if "call" not in s:
            s["call"] = _calls(s)
        return s["call"]()
    return _plain(s)


# ----------------------------------------------------------------------------- the work of a pass

def work(case):
    """Every input read once and every output written once."""
    op = case["op"]
    if op == "quantize":
        n = float(case["mats"] * case["rows"] * case["cols"])
        return {"bytes": n * ((4 if case["dtype"] == "f32" else 2) + 1 + 4.0 / (BLOCK * case["block_rows"])), "flops": 3.0 * n}
    if op == "matmul":
        rows, G, n, k = (float(case[v]) for v in ("rows", "G", "n", "k"))
        rows -= case["tail"] if case["rows"] > case["tail"] else case["rows"] - 1
        groups = min(rows, G - case["G"] // 5)  # the others are empty
        return {"bytes": (rows + groups * n / BLOCK) * k * (1 + 4.0 / BLOCK) + groups * n * k * (1 - 1.0 / BLOCK)
                         + rows * n * (4 if case["out"] == "f32" else 2), "flops": 2.0 * rows * n * k}
    if op == "moe":
        T, d, H, k, keep = case["T"], case["d"], case["H"], case["k"], case["keep"]
        active = keep * (1.0 - (1.0 - k / keep) ** T)  # experts with at least one token, expected
        weights = active * d * (_w_in_rows(case) + H)
        return {"bytes": weights * (1 + 4.0 / BLOCK**2) + 4.0 * T * d + 8.0 * T * k,
                "flops": 2.0 * T * k * d * (_w_in_rows(case) + H)}
    T, M, k = case["T"], case["M"], case["k"]
    routed = 4.0 * T * M + 4.0 * T * k + (T if case["pad"] else 0)
    if op == "balance":
        return {"bytes": routed + 8.0 * M + 4, "flops": 1.0 * T * M}
    d, R = case["d"], M + case["K"]
    eb = 4 if case["dtype"] == "f32" else 2
    return {"bytes": routed + 4.0 * T * k + (4.0 * T * M if case["full"] else 0) + 4.0 * M
                     + (2.0 * T + R) * d * eb + 4.0 * R * (d + 1), "flops": 4.0 * T * R * d}


# ----------------------------------------------------------------------------- float64 results

def _exact_round(v):
    """The nearest e4m3 value, ties to an even last digit (3 of them, 2^-9 the smallest step)."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))).clamp_min(-6.0) - 3.0)
    return (torch.round(v / step) * step).clamp(-FP8_MAX, FP8_MAX)


def _exact_quantize(x, block_rows):
    """(8-bit values as float64, float64 scales) of x [rows][cols]."""
    rows, cols = x.shape
    pad = -rows % block_rows
    b = torch.nn.functional.pad(x, (0, 0, 0, pad)).reshape((rows + pad) // block_rows, block_rows, cols // BLOCK, BLOCK)
    amax = b.abs().amax(dim=(1, 3)).clamp_min(AMAX_MIN)
    q = _exact_round(b * FP8_MAX / amax[:, None, :, None])
    return q.reshape(rows + pad, cols)[:rows], amax / FP8_MAX


def _exact_values(q, scale, block_rows):
    rows, cols = q.shape
    r = torch.arange(rows, device=DEV) // block_rows
    c = torch.arange(cols, device=DEV) // BLOCK
    return q.double() * scale.double()[r][:, c]


def _exact_expert(x, w_in, w_in_scale, w_down, w_down_scale, act):
    h = x @ _exact_values(w_in, w_in_scale, BLOCK).t()
    H = w_down.shape[1]
    h = torch.relu(h) if act == "relu" else h[:, :H] * torch.sigmoid(h[:, :H]) * h[:, H:]
    h = _exact_values(*_exact_quantize(h, 1), 1)
    return h @ _exact_values(w_down, w_down_scale, BLOCK).t()


def _exact_gate_grad(s):
    """Token by token through the softmaxes' Jacobians: with l the local and u the group logits,
    g_i = P_k p_i, dg_i/dl_j = g_i (delta_ij - p_j) inside a group, dg_i/du_k = g_i (delta - P_k)."""
    g, idx = s["probs"].double(), s["idx"].long()
    T, M = g.shape
    sel = torch.gather(g, 1, idx)
    dw = s["d_topk_w"].double()
    if s["renorm"]:
        total = sel.sum(dim=1, keepdim=True)
        dw = dw / total - (dw * sel).sum(dim=1, keepdim=True) / total.square()
    dg = s["d_balance"].double().repeat(T, 1)
    if s["d_probs"] is not None:
        dg = dg + s["d_probs"].double()
    dg = dg.scatter_add(1, idx, dw)
    if s["valid"] is not None:
        dg = dg * s["valid"][:, None]
    local, glob, at = [], [], 0
    moment = (g * dg).sum(dim=1, keepdim=True)
    for m in s["sizes"]:
        gk, dk = g[:, at:at + m], dg[:, at:at + m]
        pk = gk.sum(dim=1, keepdim=True)
        pl = gk / torch.where(pk > 0, pk, torch.ones_like(pk))
        local.append(gk * (dk - (pl * dk).sum(dim=1, keepdim=True)))
        glob.append((gk * dk).sum(dim=1, keepdim=True) - pk * moment)
        at += m
    return torch.cat(local, dim=1), torch.cat(glob, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        parts = [_exact_quantize(x.double(), case["block_rows"]) for x in s["x"]]
        return {"q": torch.stack([p[0].float() for p in parts]).to(torch.float8_e4m3fn), "scale": torch.stack([p[1] for p in parts])}
    if op == "matmul":
        out = s["out"].double()
        a = _exact_values(s["a"], s["a_scale"], 1)
        seg = [0, case["rows"]] if s["seg"] is None else s["seg"].tolist()
        for e in range(case["G"]):
            if seg[e + 1] > seg[e]:
                out[seg[e]:seg[e + 1]] = a[seg[e]:seg[e + 1]] @ _exact_values(s["b"][e], s["b_scale"][e], BLOCK).t()
        return {"out": out}
    if op == "moe":
        x = _exact_values(*_exact_quantize(s["x"].double(), 1), 1)
        y = torch.zeros_like(x)
        for e in range(case["M"]):
            t, j = torch.nonzero(s["idx"] == e, as_tuple=True)
            if t.numel():
                r = _exact_expert(x[t], s["w_in"][e], s["w_in_scale"][e], s["w_down"][e], s["w_down_scale"][e], case["act"])
                y.index_add_(0, t, r * s["w"].double()[t, j].unsqueeze(1))
        return {"y": y}
    if op == "balance":
        T, M, k = case["T"], case["M"], case["k"]
        held = torch.arange(T, device=DEV) if s["valid"] is None else torch.nonzero(s["valid"]).flatten()
        counts = torch.bincount(s["idx"][held].reshape(-1).long(), minlength=M)
        n = max(1, held.numel())
        share, mean = counts.double() / (n * k), s["probs"][held].double().sum(dim=0) / n
        return {"loss": (COEF * M * (share * mean).sum()).reshape(1), "counts": counts.to(torch.int32),
                "d_probs": COEF * M * share / n}
    local, glob = _exact_gate_grad(s)
    x = s["x"].double()
    return {"d_x": local @ s["w_local"].double() + glob @ s["w_global"].double(), "d_w_global": glob.t() @ x,
            "d_b_global": glob.sum(dim=0), "d_w_local": local.t() @ x, "d_b_local": local.sum(dim=0)}
