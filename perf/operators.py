"""The operators around a Switch FFN layer as timed cases: the dense product of a feed-forward
sublayer with its epilogue, dropout with a residual connection, and the load-balancing loss of a
router of the caller's own, each forward and backward.

A case is one call that a program makes:

  linear    switch_linear: y = residual + dropout(act(x W + bias)); with "save" also z = x W + bias
            switch_linear_backward: dx, dW and db from dy (and the saved z)
  dropout   switch_dropout: y = residual + dropout(x); its backward pass is the same call on dy
  balance   switch_balance_loss: the loss, per-expert counts and token counts
            switch_balance_loss_backward: the gradient of the logits

`listed()` names twelve of them, `draw()` gives more of the same ranges, `prepare()` makes what a
program holds before the call, `run()` makes the call or, with `own` false, computes the same in
elementary operations; `exact()` is the definition in 64 bits.

Inputs: activations and gradients ~ N(0, 1), weights ~ N(0, 1 / fan in), router logits ~ N(0, 1)
plus a spread over the experts, each rounded once to its storage type.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
ALPHA = 0.01          # coefficient of the load-balancing loss
D_LOSS = 1.0          # gradient of the loss that a training step hands down
ACTS = ("none", "relu", "gelu", "geglu")
LOW32 = 0xFFFFFFFF


# ---- cases ---------------------------------------------------------------------------------
def _linear(direction, M, K, N, act, dtype="bf16", bias=False, residual=False, dropout=0.0, save=False):
    return {"op": "linear", "direction": direction, "M": M, "K": K, "N": N, "act": act, "dtype": dtype,
            "bias": bias, "residual": residual, "dropout": dropout, "save": save}


def _dropout(rows, cols, rate, dtype="bf16", residual=True):
    return {"op": "dropout", "rows": rows, "cols": cols, "rate": rate, "dtype": dtype, "residual": residual}


def _balance(direction, T, E, k=1, groups=1, padded=0.0):
    return {"op": "balance", "direction": direction, "T": T, "E": E, "k": k, "groups": groups, "padded": padded}


def listed():
    named = [
        # One decoding step of one sequence: the gated-GELU expansion of Switch-Base's dense FFN.
        ("linear_token", _linear("forward", 1, 768, 2048, "geglu")),
        # A decoding step of 48 sequences: the contraction of the widest table entry, added to the
        # residual stream.  Reads the weights once.
        ("linear_decode", _linear("forward", 48, 10240, 4096, "none", residual=True)),
        # Prefill of an odd number of tokens: the expansion of Switch-Large's dense FFN.
        ("linear_prefill", _linear("forward", 2049, 1024, 2816, "geglu", bias=True)),
        # Training: the contraction of Switch-Base's dense FFN with dropout and residual connection.
        ("linear_train", _linear("forward", 65536, 2048, 768, "none", residual=True, dropout=0.1)),
        # Training: the ReLU expansion's backward pass, hidden dropout 0.1.
        ("linear_backward", _linear("backward", 16384, 768, 2048, "relu", bias=True, dropout=0.1)),
        # The widest gated-GELU expansion's backward pass: the largest case.
        ("linear_backward_xxl", _linear("backward", 8192, 4096, 10240, "geglu")),
        # An fp32 layer of widths that fit no tile, pre-activations kept for the backward pass ...
        ("linear_f32", _linear("forward", 3001, 1000, 520, "gelu", dtype="f32", bias=True, residual=True, save=True)),
        # ... and that backward pass.
        ("linear_f32_backward", _linear("backward", 3001, 1000, 520, "gelu", dtype="f32", bias=True)),
        # Dropout of an fp32 tensor of odd size without a residual, as a backward pass runs it.
        ("dropout_odd", _dropout(511, 1001, 0.25, dtype="f32", residual=False)),
        # Dropout on the output of a pre-training step's Switch layer, into the residual stream.
        ("dropout_block", _dropout(65536, 768, 0.1)),
        # Loss and counts of a pre-training batch, Switch-Base's experts.
        ("balance_train", _balance("forward", 65536, 128)),
        # Two choices among the most experts of the tables, padded batch in four routing groups.
        ("balance_wide_backward", _balance("backward", 16384, 2048, k=2, groups=4, padded=0.2)),
    ]
    return [dict(case, name=name) for name, case in named]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more call: 1 .. 65536 rows, widths 64 .. 10240, 2 .. 4096 experts, every option."""
    kind = rng.choices(("linear", "dropout", "balance"), (6, 2, 2))[0]
    while True:
        if kind == "linear":
            dtype = rng.choices(("bf16", "f32"), (7, 3))[0]
            step = 8 if dtype == "bf16" else 4
            direction = rng.choice(("forward", "backward"))
            act = rng.choice(ACTS)
            case = _linear(direction, round(_log_uniform(rng, 1, 65536)), step * round(_log_uniform(rng, 64, 10240) / step),
                           step * round(_log_uniform(rng, 64, 10240) / step), act, dtype=dtype, bias=rng.random() < 0.5,
                           residual=direction == "forward" and rng.random() < 0.4, dropout=rng.choice((0.0, 0.0, 0.1, 0.25)),
                           save=direction == "forward" and act != "none" and rng.random() < 0.4)
            most = 2.6e12 if dtype == "bf16" else 1.5e11
            if work(case)["flops"] > most or work(case)["bytes"] > 1.5e9:
                continue
            return case
        if kind == "dropout":
            case = _dropout(round(_log_uniform(rng, 1, 65536)), round(_log_uniform(rng, 64, 10240)), rng.choice((0.1, 0.25, 0.5)),
                            dtype=rng.choice(("bf16", "f32")), residual=rng.random() < 0.5)
            if case["rows"] * case["cols"] <= 65536 * 768:
                return case
            continue
        E = round(_log_uniform(rng, 2, 4096))
        groups = rng.choice((1, 1, 2, 8))
        T = groups * max(1, round(_log_uniform(rng, 1, 65536) / groups))
        if T * E <= 65536 * 512:
            return _balance(rng.choice(("forward", "backward")), T, E, k=rng.randint(1, min(E, 4)), groups=groups,
                            padded=rng.choice((0.0, 0.0, 0.1, 0.5)))


def _z_columns(case):
    return case["N"] * (2 if case["act"] == "geglu" else 1)


# ---- what a program holds before the call ----------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)

    def normal(*size):
        return torch.randn(size, generator=gen, device=DEVICE)

    state = {"case": case, "seed": 17 + seed}
    if case["op"] == "linear":
        M, K, N, Nz, dt = case["M"], case["K"], case["N"], _z_columns(case), _dtype(case)
        state["x"] = normal(M, K).to(dt)
        state["W"] = normal(K, Nz).mul_(K ** -0.5).to(dt)
        state["bias"] = normal(Nz) * 0.1 if case["bias"] else None
        if case["direction"] == "forward":
            state["residual"] = normal(M, N).to(dt) if case["residual"] else None
        else:
            state["dy"] = normal(M, N).to(dt)
            z = None
            if case["act"] != "none":   # as the forward pass left it, to the rounding of its sums
                z = state["x"] @ state["W"]
                z = z if state["bias"] is None else (z + state["bias"]).to(dt)
            state["z"] = z
    elif case["op"] == "dropout":
        state["x"] = normal(case["rows"], case["cols"]).to(_dtype(case))
        state["residual"] = normal(case["rows"], case["cols"]).to(_dtype(case)) if case["residual"] else None
    else:
        T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
        logits = normal(T, E) + 0.5 * normal(E)
        index = torch.topk(logits, k, dim=1).indices.to(torch.int32)
        mask = None
        if case["padded"] > 0.0:   # the tails of 512-token sequences; what stands there means nothing
            place = torch.arange(T, device=DEVICE) % 512
            mask = (place < 512 * (1.0 - case["padded"])).to(torch.uint8)
            logits[mask == 0] = float("nan")
            index[mask == 0] = -1
        state.update(logits=logits, index=index, mask=mask)
        if case["direction"] == "backward":
            state["counts"], state["tokens"] = _counts(case, index, mask)
    return state


def _counts(case, index, mask):
    """Choices per group and expert, tokens per group that are not padding."""
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    group = torch.arange(T, device=DEVICE) // (T // groups)
    valid = torch.ones(T, dtype=torch.bool, device=DEVICE) if mask is None else mask != 0
    # an extra cell takes the choices that do not count
    cell = torch.where(valid[:, None] & (index >= 0) & (index < E), group[:, None] * E + index, groups * E)
    counts = torch.bincount(cell.reshape(-1), minlength=groups * E + 1)[:groups * E].reshape(groups, E)
    return counts.to(torch.int32), valid.reshape(groups, -1).sum(1).to(torch.int32)


def prepare(case, seed):
    state = _inputs(case, seed)

    def empty(*size, dtype=torch.float32):
        return torch.empty(size, dtype=dtype, device=DEVICE)

    if case["op"] == "linear":
        M, K, N, Nz, dt = case["M"], case["K"], case["N"], _z_columns(case), _dtype(case)
        if case["direction"] == "forward":
            state["out"] = {"y": empty(M, N, dtype=dt)}
            if case["save"]:
                state["out"]["z"] = empty(M, Nz, dtype=dt)
        else:
            state["out"] = {"dx": empty(M, K, dtype=dt), "dW": empty(K, Nz, dtype=dt)}
            if case["bias"]:
                state["out"]["db"] = empty(Nz)
    elif case["op"] == "dropout":
        state["out"] = {"y": torch.empty_like(state["x"])}
    elif case["direction"] == "forward":
        state["out"] = {"loss": empty(1), "counts": empty(case["groups"], case["E"], dtype=torch.int32),
                        "tokens": empty(case["groups"], dtype=torch.int32)}
    else:
        state["out"] = {"dlogits": torch.empty_like(state["logits"])}
    return state


# ---- one pass ----------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "linear":
        return (_linear_forward if case["direction"] == "forward" else _linear_backward)(case, state)
    if case["op"] == "dropout":
        x = state["x"]
        y = x.float() * _dropout_factor(x.shape, case["rate"], state["seed"])
        return {"y": (y if state["residual"] is None else y + state["residual"].float()).to(x.dtype)}
    return (_balance_forward if case["direction"] == "forward" else _balance_backward)(case, state)


def _run_own(case, state):
    import paper_2101_03961_amd as sw
    stream = torch.cuda.current_stream().cuda_stream
    out = state["out"]
    dtype = sw.SW_F32 if case.get("dtype") == "f32" else sw.SW_BF16
    if case["op"] == "dropout":
        x = state["x"]
        sw.switch_dropout(x.numel(), dtype, case["rate"], state["seed"], x, state["residual"], out["y"], stream)
        return out
    if "call" not in state:   # the configuration and workspace that a program keeps
        if case["op"] == "linear":
            cfg = sw.SwitchLinearConfig(case["M"], case["K"], case["N"], dtype, ACTS.index(case["act"]), case["dropout"], 0,
                                        state["seed"])
            size = sw.switch_linear_workspace_size(cfg, case["direction"] == "backward")
        else:
            cfg = sw.SwitchBalanceConfig(case["T"], case["E"], case["k"], case["groups"], ALPHA, 0)
            size = sw.switch_balance_workspace_size(cfg)
        state["call"] = cfg, torch.empty(max(size, 1), dtype=torch.uint8, device=DEVICE), size
    cfg, workspace, size = state["call"]
    if case["op"] == "linear" and case["direction"] == "forward":
        sw.switch_linear(cfg, state["x"], state["W"], state["bias"], state["residual"], out["y"], out.get("z"), workspace,
                         size, stream)
    elif case["op"] == "linear":
        sw.switch_linear_backward(cfg, state["dy"], state["x"], state["W"], state["z"], out["dx"], out["dW"], out.get("db"),
                                  workspace, size, stream)
    elif case["direction"] == "forward":
        sw.switch_balance_loss(cfg, state["logits"], state["index"], state["mask"], out["loss"], out["counts"],
                               out["tokens"], workspace, size, stream)
    else:
        sw.switch_balance_loss_backward(cfg, D_LOSS, state["logits"], state["mask"], state["counts"], state["tokens"],
                                        out["dlogits"], stream)
    return out


def _threshold(rate):
    return math.floor(float(np.float32(rate)) * 65536.0)


def _dropout_factor(shape, rate, seed):
    """0 or 1 / (1 - rate) of each element: the library's generator, stream 3, two elements a draw."""
    n = math.prod(shape)
    thr = _threshold(rate)
    pair = torch.arange((n + 1) // 2, device=DEVICE)
    term = ((seed >> 32) + 3 * 0x7F4A7C15) & LOW32
    z = (((pair & LOW32) ^ (seed & LOW32)) * 0x9E3779B1) & LOW32
    z ^= z >> 15
    z = ((z + term + (pair >> 32) * 0x632BE5AB) * 0x85EBCA77) & LOW32
    z ^= z >> 13
    z = (z * 0xC2B2AE3D) & LOW32
    z ^= z >> 16
    keep = torch.stack(((z & 0xFFFF) >= thr, (z >> 16) >= thr), dim=1).reshape(-1)[:n].reshape(shape)
    return keep * (65536.0 / (65536.0 - thr))


def _phi(u):
    """Distribution function of the standard normal distribution."""
    return 0.5 * torch.erfc(u * -math.sqrt(0.5))


def _linear_forward(case, state):
    dt, N = _dtype(case), case["N"]
    z = state["x"].float() @ state["W"].float()
    if state["bias"] is not None:
        z = z + state["bias"]
    if case["act"] == "geglu":
        y = z[:, :N] * _phi(z[:, :N]) * z[:, N:]
    elif case["act"] == "gelu":
        y = z * _phi(z)
    else:
        y = torch.clamp(z, min=0.0) if case["act"] == "relu" else z
    if case["dropout"] > 0.0:
        y = y * _dropout_factor(y.shape, case["dropout"], state["seed"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return {"y": y.to(dt), "z": z.to(dt)} if case["save"] else {"y": y.to(dt)}


def _linear_backward(case, state):
    dt, N = _dtype(case), case["N"]
    d = state["dy"].float()
    if case["dropout"] > 0.0:
        d = d * _dropout_factor(d.shape, case["dropout"], state["seed"])
    if case["act"] == "relu":
        d = torch.where(state["z"] > 0, d, 0.0)
    elif case["act"] != "none":
        z = state["z"].float()
        u = z[:, :N]
        cdf = _phi(u)
        slope = cdf + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
        d = torch.cat((d * z[:, N:] * slope, d * u * cdf), dim=1) if case["act"] == "geglu" else d * slope
    out = {"dx": (d @ state["W"].float().t()).to(dt), "dW": (state["x"].float().t() @ d).to(dt)}
    if case["bias"]:
        out["db"] = d.sum(0)
    return out


def _probabilities(state):
    """Softmax of each row; rows of padding are zero."""
    h = state["logits"]
    if state["mask"] is not None:
        h = torch.where(state["mask"][:, None] != 0, h, 0.0)
    e = torch.exp(h - h.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    return p if state["mask"] is None else torch.where(state["mask"][:, None] != 0, p, 0.0)


def _balance_forward(case, state):
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    counts, tokens = _counts(case, state["index"], state["mask"])
    n = tokens.double().clamp(min=1.0)[:, None]
    f = counts.double() / (n * k)
    P = _probabilities(state).reshape(groups, T // groups, E).sum(1).double() / n
    loss = ALPHA * E * (f * P).sum() / groups
    return {"loss": loss.float().reshape(1), "counts": counts, "tokens": tokens}


def _balance_backward(case, state):
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    n = state["tokens"].double().clamp(min=1.0)[:, None]
    f = state["counts"].double() / (n * k)
    # the mean over the experts drops out of the gradient: taken off first, where little is lost to it
    c = (D_LOSS * ALPHA * E / groups * (f - f.mean(1, keepdim=True)) / n).float()
    p = _probabilities(state).reshape(groups, T // groups, E)
    c = c[:, None, :]
    return {"dlogits": (p * (c - (p * c).sum(2, keepdim=True))).reshape(T, E)}


# ---- the definition in 64 bits -------------------------------------------------------------------
def _exact_keep(n, rate, seed):
    """The generator's decisions in 32-bit words that wrap by themselves."""
    pair = np.arange((n + 1) // 2, dtype=np.uint64)
    z = (pair.astype(np.uint32) ^ np.uint32(seed & LOW32)) * np.uint32(0x9E3779B1)
    z ^= z >> np.uint32(15)
    z += np.uint32(((seed >> 32) + 3 * 0x7F4A7C15) & LOW32)
    z += (pair >> np.uint64(32)).astype(np.uint32) * np.uint32(0x632BE5AB)
    z *= np.uint32(0x85EBCA77)
    z ^= z >> np.uint32(13)
    z *= np.uint32(0xC2B2AE3D)
    z ^= z >> np.uint32(16)
    halves = z.astype("<u4", copy=False).view("<u2")[:n]   # low half first
    return torch.from_numpy(halves >= _threshold(rate)).to(DEVICE)


def _exact_dropout(t, rate, seed):
    keep = _exact_keep(t.numel(), rate, seed).reshape(t.shape)
    return torch.where(keep, t, 0.0) / (1.0 - _threshold(rate) / 65536.0)


def _exact_gelu(u):
    return u * torch.special.ndtr(u)


def _exact_gelu_slope(u):
    return torch.special.ndtr(u) + u * torch.exp(-u.square() / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = _inputs(case, seed)
    s64 = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"] == "dropout":
        y = _exact_dropout(s64["x"], case["rate"], s["seed"])
        return {"y": y if s["residual"] is None else s64["residual"] + y}
    if case["op"] == "linear":
        N, act, rate = case["N"], case["act"], case["dropout"]
        if case["direction"] == "forward":
            z = torch.mm(s64["x"], s64["W"])
            if s["bias"] is not None:
                z += s64["bias"]
            y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0), "gelu": lambda: _exact_gelu(z),
                 "geglu": lambda: _exact_gelu(z[:, :N]) * z[:, N:]}[act]()
            if rate > 0.0:
                y = _exact_dropout(y, rate, s["seed"])
            if s["residual"] is not None:
                y = s64["residual"] + y
            return {"y": y, "z": z} if case["save"] else {"y": y}
        g = s64["dy"] if rate == 0.0 else _exact_dropout(s64["dy"], rate, s["seed"])
        z = s64["z"]
        if act == "relu":
            g = g * (z > 0)
        elif act == "gelu":
            g = g * _exact_gelu_slope(z)
        elif act == "geglu":
            gate, linear = z.split(N, dim=1)
            g = torch.cat((g * linear * _exact_gelu_slope(gate), g * _exact_gelu(gate)), dim=1)
        out = {"dx": torch.mm(g, s64["W"].t().contiguous()), "dW": torch.mm(s64["x"].t().contiguous(), g)}
        if case["bias"]:
            out["db"] = g.sum(0)
        return out
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    valid = torch.ones(T, 1, dtype=torch.bool, device=DEVICE) if s["mask"] is None else s["mask"].bool()[:, None]
    h = s64["logits"].masked_fill(~valid, 0.0)
    p = torch.exp(h - torch.logsumexp(h, 1, keepdim=True)).masked_fill(~valid, 0.0).reshape(groups, -1, E)
    counts, tokens = _counts(case, s["index"], s["mask"])
    n = tokens.double().clamp(min=1.0).reshape(groups, 1)
    f = counts.double() / n / k
    if case["direction"] == "forward":
        return {"loss": (ALPHA * E / groups * (f * p.sum(1) / n).sum()).reshape(1), "counts": counts, "tokens": tokens}
    dp = (D_LOSS * ALPHA * E / groups * f / n)[:, None, :]
    return {"dlogits": (p * (dp - (p * dp).sum(2, keepdim=True))).reshape(T, E)}


def work(case):
    """Every input read once, every output written once; multiplications and additions of the products."""
    if case["op"] == "linear":
        M, K, N, Nz = case["M"], case["K"], case["N"], _z_columns(case)
        elt = 2 if case["dtype"] == "bf16" else 4
        bias = 4 * Nz if case["bias"] else 0
        if case["direction"] == "forward":
            nbytes = elt * (M * K + K * Nz + M * N * (2 if case["residual"] else 1) + (M * Nz if case["save"] else 0)) + bias
            return {"bytes": float(nbytes), "flops": 2.0 * M * K * Nz}
        nbytes = elt * (2 * M * K + 2 * K * Nz + M * N + (M * Nz if case["act"] != "none" else 0)) + bias
        return {"bytes": float(nbytes), "flops": 4.0 * M * K * Nz}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": float(n * (2 if case["dtype"] == "bf16" else 4) * (3 if case["residual"] else 2)), "flops": 3.0 * n}
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    live = T * (1.0 - case["padded"])
    padding = T if case["padded"] > 0.0 else 0
    if case["direction"] == "forward":
        return {"bytes": 4.0 * live * (E + k) + padding + 4.0 * groups * (E + 1), "flops": 4.0 * live * E}
    return {"bytes": 4.0 * E * (live + T) + padding + 4.0 * groups * (E + 1), "flops": 8.0 * live * E}
