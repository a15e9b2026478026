"""The training-side operators and how they are measured: gradients of the dictionary regression, the balance loss of a
per-pixel selection with its gradient, and the AdamW step over many tensors.

`listed()` and `draw()` give cases, `prepare()` a case's inputs on the GPU, `run()` one pass, either in plain torch operations
or (with `own` set) through the library's calls, `exact()` the same results in 64 bits, `work()` the bytes and operations a pass
cannot do without.
"""
import math

import torch

own = False

UPSAMPLE_BILINEAR = 8
IDX_GLOBAL, COEF_COMPACT = 2, 4
GRAD_ADD, BALANCE_PER_FRAME = 128, 256
QUANT_BLOCK = 256            # elements that share one scale of an 8-bit optimiser state
F8_MAX = 448.0               # largest e4m3 value


# ---- cases -------------------------------------------------------------------------------------------------------------

def _grad(name, mode, dtype, n, c, h, w, scale, D, k, s=0, bilinear=False):
    return {"name": name, "op": "grad", "mode": mode, "dtype": dtype, "n": n, "c": c, "h": h, "w": w, "scale": scale, "D": D, "k": k,
            "s": s, "bilinear": bilinear}


def _balance(name, dtype, n, H, W, D, s, per_frame=False, masked=False, add=False):
    return {"name": name, "op": "balance", "dtype": dtype, "n": n, "H": H, "W": W, "D": D, "s": s, "per_frame": per_frame,
            "masked": masked, "add": add}


def _adamw(name, tensors, smallest, largest, param, grad, bits):
    return {"name": name, "op": "adamw", "tensors": tensors, "smallest": smallest, "largest": largest, "param": param, "grad": grad, "bits": bits}


def listed():
    return [
        # a patch of a training batch in fp32: the smallest call, latency
        _grad("grad f32 64x64 x2", "dense", "f32", 1, 3, 64, 64, 2, 72, 5),
        # the headline frame, every atom: one full-HD frame of a fine-tuning step
        _grad("grad f16 1080p x4", "dense", "f16", 1, 3, 270, 480, 4, 72, 5),
        # a batch of four 4K frames: the largest call, element offsets beyond 2^31
        _grad("grad f16 4K x2 batch", "dense", "f16", 4, 3, 1080, 1920, 2, 72, 5),
        # the headline frame under per-pixel selection: gradients reach the listed atoms only
        _grad("grad lists 1080p x4", "listed", "f16", 1, 3, 270, 480, 4, 72, 5, 8),
        # kept values alone (compact planes), odd frame, 7 x 7 atoms at scale 3, up-sampled bilinearly: no size a multiple of a tile
        _grad("grad compact odd x3", "compact", "f16", 2, 3, 93, 131, 3, 32, 7, 4, True),
        # the subset a selection search left, with its re-weights: the fine-tuning that follows the search
        _grad("grad subset 1080p x4", "global", "f16", 1, 3, 270, 480, 4, 72, 5, 8),
        # the selection's balance on the headline frame, added to the regression's gradient
        _balance("balance f16 1080p", "f16", 1, 1080, 1920, 72, 8, add=True),
        # padded training patches of odd size, each balanced by itself, fp32
        _balance("balance f32 patches", "f32", 8, 95, 127, 72, 8, per_frame=True, masked=True),
        # one small binary16 patch, few atoms: latency
        _balance("balance f16 128x128", "f16", 1, 128, 128, 32, 4),
        # the dictionary and the last layer (weights and bias) of the headline configuration
        _adamw("adamw last layer", 3, 1152, 331776, "f32", "f32", 32),
        # a network's many small and odd tensors, binary16 gradients, 8-bit states
        _adamw("adamw 8-bit many", 160, 1, 400001, "f32", "f16", 8),
        # a large network, states in 32 bits
        _adamw("adamw 32-bit large", 24, 100000, 12000000, "f32", "f32", 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["grad", "grad", "grad", "balance", "adamw"])
    if op == "adamw":
        largest = _log_int(rng, 300, 12000000)
        return {"op": "adamw", "tensors": _log_int(rng, 1, 200) if largest < 500000 else _log_int(rng, 1, 24),
                "smallest": max(1, largest // _log_int(rng, 1, 5000)), "largest": largest, "param": rng.choice(["f32", "f32", "f16", "bf16"]),
                "grad": rng.choice(["f32", "f16", "bf16"]), "bits": rng.choice([8, 32])}
    dtype = rng.choice(["f16", "f16", "f32"])
    D = _log_int(rng, 8, 128)
    s = min(D, rng.randint(1, 16))
    pixels = _log_int(rng, 4000, 6000000 if dtype == "f16" else 2000000)
    n = rng.choice([1, 1, 2, 3])
    if op == "balance":
        H = max(8, int(math.sqrt(pixels / n) * rng.uniform(0.5, 1.5)))
        W = max(8, int(pixels / n / H))
        return {"op": "balance", "dtype": dtype, "n": n, "H": H, "W": W, "D": D, "s": s, "per_frame": rng.random() < 0.5,
                "masked": rng.random() < 0.5, "add": rng.random() < 0.5}
    scale = rng.choice([1, 2, 3, 4])
    h = max(4, int(math.sqrt(pixels / n) * rng.uniform(0.5, 1.5) / scale))
    w = max(4, int(pixels / n / scale / scale / h))
    if rng.random() < 0.6:
        w = (w + 7) // 8 * 8
    mode = rng.choice(["dense", "dense", "listed", "compact", "global"])
    return {"op": "grad", "mode": mode, "dtype": dtype, "n": n, "c": rng.choice([1, 3, 3]), "h": h, "w": w, "scale": scale, "D": D,
            "k": rng.choice([3, 5, 5, 7]), "s": 0 if mode == "dense" else s, "bilinear": rng.random() < 0.25}


# ---- inputs ------------------------------------------------------------------------------------------------------------

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _normal(shape, gen, mean=0.0, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=gen)


def _top(coef, s):
    """The s atoms of largest magnitude at every pixel, in rank order, ties to the lower atom (a stable sort)."""
    key = coef.abs().permute(0, 2, 3, 1).reshape(-1, coef.shape[1])
    parts = [torch.sort(part, dim=1, descending=True, stable=True).indices[:, :s].to(torch.uint8) for part in key.split(1 << 20)]
    n, _, H, W = coef.shape
    return torch.cat(parts).reshape(n, H, W, s).permute(0, 3, 1, 2).contiguous()


def _adamw_sizes(case):
    """Sizes from the smallest to the largest, evenly spread over their logarithm, every third one odd."""
    t, lo, hi = case["tensors"], case["smallest"], case["largest"]
    sizes = [int(round(lo * (hi / lo) ** (i / max(1, t - 1)))) for i in range(t)]
    return [hi if t == 1 else (x | 1 if i % 3 == 1 else x) for i, x in enumerate(sizes)]


def _spread(sizes, unit):
    """Where each tensor starts in one buffer, each at a multiple of `unit`, and the buffer's length."""
    starts, at = [], 0
    for x in sizes:
        starts.append(at)
        at += (x + unit - 1) // unit * unit
    return starts, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen)
    dtype, D = _DTYPES[case["dtype"]], case["D"]
    if case["op"] == "balance":
        n, H, W = case["n"], case["H"], case["W"]
        coef = _normal((n, D, H, W), gen, 1.0 / D, 0.05, dtype)
        coef[:, : max(1, D // 8)] *= 3.0                       # some atoms are chosen far more often than others
        mask = None
        if case["masked"]:                                     # padded frames: the right and the lower margin do not count
            rows = torch.randint(H // 2, H + 1, (n, 1, 1), generator=gen, device="cuda")
            cols = torch.randint(W // 2, W + 1, (n, 1, 1), generator=gen, device="cuda")
            y, x = torch.arange(H, device="cuda").view(1, H, 1), torch.arange(W, device="cuda").view(1, 1, W)
            mask = ((y < rows) & (x < cols)).to(torch.uint8).contiguous()
        grad = _normal((n, D, H, W), gen, 0.0, 0.01, dtype) if case["add"] else torch.empty_like(coef)
        # the weight holds a loss scale that brings 1 / pixels into the range of binary16
        return {"case": case, "coef": coef, "idx": _top(coef, case["s"]), "mask": mask, "grad": grad, "weight": 0.01 * n * H * W}
    n, c, h, w, r, k, s = (case[x] for x in ("n", "c", "h", "w", "scale", "k", "s"))
    H, W = h * r, w * r
    lr = torch.empty((n, c, h, w), device="cuda").uniform_(generator=gen)
    coef = _normal((n, D, H, W), gen, 1.0 / D, 0.05, dtype)
    ax = torch.arange(k, device="cuda") - (k - 1) / 2
    sigma = torch.empty((D, 1, 1), device="cuda").uniform_(0.3, 2.0, generator=gen)
    atoms = torch.exp(-(ax.view(1, k, 1) ** 2 + ax.view(1, 1, k) ** 2) / (2 * sigma * sigma)).reshape(D, k * k)
    dict_ = (atoms / atoms.sum(1, keepdim=True) + _normal((D, k * k), gen, 0.0, 0.02)).contiguous()
    state = {"case": case, "lr": lr, "dict": dict_, "grad_out": _normal((n, c, H, W), gen, 0.0, 0.02), "coef": coef, "idx": None, "gamma": None}
    if case["mode"] in ("listed", "compact"):
        state["idx"] = _top(coef, s)
    if case["mode"] == "compact":
        state["coef"] = torch.gather(coef, 1, state["idx"].long()).contiguous()
    if case["mode"] == "global":
        state["idx"] = torch.randperm(D, generator=gen, device="cuda")[:s].sort().values.to(torch.uint8)
        state["gamma"] = torch.empty(s, device="cuda").uniform_(0.5, 1.5, generator=gen)
    return state


def _prepare_adamw(case, gen):
    sizes = _adamw_sizes(case)
    starts, total = _spread(sizes, QUANT_BLOCK)                # 256 elements: one scale of the 8-bit states per block of the buffer
    at = lambda buf, unit=1: [buf[a // unit: a // unit + (x + unit - 1) // unit] for a, x in zip(starts, sizes)]  # noqa: E731
    where = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, x in zip(starts, sizes):
        where[a: a + x] = True
    spread = torch.exp(_normal(((total + 1023) // 1024,), gen, -4.0, 1.5)).repeat_interleave(1024)[:total]   # layers differ in their gradients' size
    param = (_normal((total,), gen, 0.0, 0.05) * where).to(_DTYPES[case["param"]])
    grad = (_normal((total,), gen) * spread * where).to(_DTYPES[case["grad"]])
    m = _normal((total,), gen) * spread * 0.3 * where
    root_v = (_normal((total,), gen).abs() + 0.2) * spread * where
    state = {"case": case, "param": param, "grad": grad, "sizes": sizes, "step": 100,
             "opts": {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "grad_scale": 0.5}}
    if case["bits"] == 8:
        state["m_scale"], state["v_scale"] = (x.view(-1, QUANT_BLOCK).abs().amax(1) / F8_MAX for x in (m, root_v))
        state["m"], state["v"] = (_e4m3(x.view(-1, QUANT_BLOCK), q).view(-1) for x, q in ((m, state["m_scale"]), (root_v, state["v_scale"])))
        state["m_scales"], state["v_scales"] = at(state["m_scale"], QUANT_BLOCK), at(state["v_scale"], QUANT_BLOCK)
    else:
        state["m"], state["v"] = m, root_v * root_v
        state["m_scales"] = state["v_scales"] = None
    for name in ("param", "grad", "m", "v"):
        state[name + "s"] = at(state[name])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"grad": _own_grad, "balance": _own_balance, "adamw": _own_adamw}[op](state)
    return {"grad": _plain_grad, "balance": _plain_balance, "adamw": _plain_adamw}[op](state)


def _own_grad(state):
    import paper_2303_08999_b200 as sr
    case, flags = state["case"], UPSAMPLE_BILINEAR if state["case"]["bilinear"] else 0
    if case["mode"] == "dense":
        return sr.sr_dict_regress_dense_grad(state["lr"], state["coef"], state["dict"], state["grad_out"], case["scale"], case["k"], flags)
    flags |= {"listed": 0, "compact": COEF_COMPACT, "global": IDX_GLOBAL}[case["mode"]]
    return sr.sr_dict_regress_selected_grad(state["lr"], state["coef"], state["idx"], state["gamma"], state["dict"], state["grad_out"],
                                            case["scale"], case["k"], case["s"], flags)


def _own_balance(state):
    import paper_2303_08999_b200 as sr
    case = state["case"]
    loss, counts, share, slope = sr.sr_select_balance(state["coef"], state["idx"], state["mask"], BALANCE_PER_FRAME if case["per_frame"] else 0)
    grad = sr.sr_select_balance_grad(state["coef"], slope, state["mask"], state["weight"], flags=GRAD_ADD if case["add"] else 0,
                                     grad_coef=state["grad"])
    return loss, counts, share, slope, grad


def _own_adamw(state):
    import paper_2303_08999_b200 as sr
    if "plan" not in state:                                    # the handle that an optimiser keeps for its tensors
        state["plan"] = sr.sr_adamw_plan(state["params"], state["ms"], state["vs"], state["m_scales"], state["v_scales"])
    sr.sr_adamw_step(state["plan"], state["grads"], state["step"], **state["opts"])
    return _adamw_outputs(state)


def _adamw_outputs(state):
    return [state["param"], state["m"], state["v"]] + ([state["m_scale"], state["v_scale"]] if state["case"]["bits"] == 8 else [])


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _taps(size, scale, bilinear):
    """For every HR coordinate of an axis its four LR indices (clamped) and weights: Keys cubic convolution with a = -0.75 at half-pixel
    centres, or the linear pair in the two middle taps."""
    src = (torch.arange(size * scale, device="cuda", dtype=torch.float64) + 0.5) / scale - 0.5
    base = torch.floor(src)
    t = src - base
    dist = torch.stack([t + 1, t, 1 - t, 2 - t], 1)
    near = (1.25 * dist - 2.25) * dist * dist + 1
    far = ((-0.75 * dist + 3.75) * dist - 6.0) * dist + 3.0
    weight = torch.clamp(1 - dist, min=0) if bilinear else torch.where(dist <= 1, near, far)
    at = torch.clamp(base.long().view(-1, 1) + torch.arange(-1, 3, device="cuda"), 0, size - 1)
    return at, weight.float()


def _patch_grad(state):
    """G [n][H][W][k*k]: sum over channels of the output's gradient times the up-sampled patch."""
    case, g = state["case"], state["grad_out"]
    n, c, h, w, r, k = (case[x] for x in ("n", "c", "h", "w", "scale", "k"))
    (ay, wy), (ax, wx) = _taps(h, r, case["bilinear"]), _taps(w, r, case["bilinear"])
    u = (state["lr"][:, :, ay] * wy.view(1, 1, h * r, 4, 1)).sum(3)
    u = (u[:, :, :, ax] * wx.view(1, 1, 1, w * r, 4)).sum(4)
    p = (k - 1) // 2
    rows = torch.clamp(torch.arange(-p, h * r + p, device="cuda"), 0, h * r - 1)
    cols = torch.clamp(torch.arange(-p, w * r + p, device="cuda"), 0, w * r - 1)
    patches = u[:, :, rows][:, :, :, cols].unfold(2, k, 1).unfold(3, k, 1)
    return (patches * g[..., None, None]).sum(1).flatten(3)


def _atom_sums(weights, G):
    """[planes][k*k]: sum over frames and pixels of weights [n][planes][H][W] times G; rows in 32 bits, their sum in 64."""
    return torch.matmul(weights.permute(0, 2, 1, 3), G).sum((0, 1), dtype=torch.float64)


def _plain_grad(state):
    case, coef, dict_, idx = state["case"], state["coef"], state["dict"], state["idx"]
    n, H, W, D = case["n"], case["h"] * case["scale"], case["w"] * case["scale"], case["D"]
    G = _patch_grad(state)
    if case["mode"] == "global":
        atoms, gamma = idx.long(), state["gamma"]
        d_atoms = _atom_sums(coef[:, atoms].float(), G)
        g_coef = torch.zeros_like(coef)
        g_coef[:, atoms] = torch.matmul(G, (gamma.view(-1, 1) * dict_[atoms]).t()).permute(0, 3, 1, 2).to(coef.dtype)
        g_dict = torch.zeros_like(dict_)
        g_dict[atoms] = (gamma.view(-1, 1) * d_atoms).float()
        return g_coef, g_dict, (dict_[atoms] * d_atoms).sum(1).float()
    full = torch.matmul(G, dict_.t()).permute(0, 3, 1, 2)
    if case["mode"] == "dense":
        return full.to(coef.dtype, memory_format=torch.contiguous_format), _atom_sums(coef.float(), G).float()
    at = idx.long()
    if case["mode"] == "compact":
        weights = torch.zeros((n, D, H, W), device="cuda").scatter_(1, at, coef.float())
        return torch.gather(full, 1, at).to(coef.dtype, memory_format=torch.contiguous_format), _atom_sums(weights, G).float(), None
    keep = torch.zeros((n, D, H, W), device="cuda").scatter_(1, at, 1.0)
    g_coef = (full * keep).to(coef.dtype, memory_format=torch.contiguous_format)
    return g_coef, _atom_sums(coef.float() * keep, G).float(), None


def _plain_balance(state):
    case, coef, idx, mask = state["case"], state["coef"], state["idx"], state["mask"]
    n, H, W, D, s = (case[x] for x in ("n", "H", "W", "D", "s"))
    value = coef.float()
    on = torch.ones((n, 1, H, W), device="cuda") if mask is None else mask.float().unsqueeze(1)
    total = value.abs().sum(1, keepdim=True)
    p = torch.where(total > 0, value.abs() / total, 1.0 / D) * on
    counts = torch.zeros((n, D), dtype=torch.int64, device="cuda").scatter_add_(1, idx.flatten(1).long(), on.long().expand(n, s, H, W).flatten(1))
    valid = on.sum((1, 2, 3), dtype=torch.float64)
    sums = p.sum((2, 3), dtype=torch.float64)
    share = sums / valid.clamp(min=1).view(n, 1)
    if case["per_frame"]:
        a = D * counts / (s * n * valid.clamp(min=1).view(n, 1) ** 2)
    else:
        a = (D * counts.sum(0, keepdim=True) / (s * valid.sum().clamp(min=1) ** 2)).expand(n, D)
    loss = (a * sums).sum()
    a = a.float().view(n, D, 1, 1)
    grad = state["weight"] * torch.sign(value) * (a - (a * p).sum(1, keepdim=True)) / total * on
    grad = torch.where(total > 0, grad, 0.0)
    state["grad"].copy_(state["grad"].float() + grad if case["add"] else grad)
    return loss.float().view(1), counts.int(), share.float(), a.view(n, D), state["grad"]


def _e4m3(x, scale):
    """x [blocks][256] over its block's scale, rounded to e4m3; 0 where the scale is 0."""
    return torch.where(scale.view(-1, 1) > 0, x / scale.view(-1, 1), 0.0).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)


def _plain_adamw(state):
    """On the whole buffers at once: the gaps between the tensors hold zeros, which the step leaves zeros, and share no block of 256."""
    o, t, eight = state["opts"], state["step"], state["case"]["bits"] == 8
    p, g = state["param"].float(), state["grad"].float() * o["grad_scale"]
    m, v = state["m"].float(), state["v"].float()
    if eight:
        m = (m.view(-1, QUANT_BLOCK) * state["m_scale"].view(-1, 1)).view(-1)
        v = (v.view(-1, QUANT_BLOCK) * state["v_scale"].view(-1, 1)).view(-1) ** 2
    m = o["beta1"] * m + (1 - o["beta1"]) * g
    v = o["beta2"] * v + (1 - o["beta2"]) * (g * g)
    denom = torch.sqrt(v) / math.sqrt(1 - o["beta2"] ** t) + o["eps"]
    p = p * (1 - o["lr"] * o["weight_decay"]) - o["lr"] / (1 - o["beta1"] ** t) * (m / denom)
    state["param"].copy_(p)
    if eight:
        m, root = m.view(-1, QUANT_BLOCK), torch.sqrt(v).view(-1, QUANT_BLOCK)
        state["m_scale"].copy_(m.abs().amax(1) / F8_MAX)
        state["v_scale"].copy_(root.amax(1) / F8_MAX)
        code_v = _e4m3(root, state["v_scale"]).float()
        code_v = torch.where((root > 0) & (code_v == 0) & (state["v_scale"].view(-1, 1) > 0), 2.0 ** -9, code_v)   # a root that is not zero is not held as zero
        state["m"].copy_(_e4m3(m, state["m_scale"]).view(-1))
        state["v"].copy_(code_v.to(torch.float8_e4m3fn).view(-1))
    else:
        state["m"].copy_(m)
        state["v"].copy_(v)
    return _adamw_outputs(state)


# ---- 64 bits -----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    return {"grad": _exact_grad, "balance": _exact_balance, "adamw": _exact_adamw}[case["op"]](state)


def _matrix(size, scale, bilinear):
    """[HR][LR] up-sampling matrix of an axis."""
    def cubic(x):
        x = abs(x)
        if x <= 1:
            return 1.25 * x ** 3 - 2.25 * x ** 2 + 1
        return -0.75 * x ** 3 + 3.75 * x ** 2 - 6 * x + 3 if x < 2 else 0.0
    rows, cols, values = [], [], []
    for X in range(size * scale):
        src = (2 * X + 1 - scale) / (2 * scale)
        for q in range(math.floor(src) - 1, math.floor(src) + 3):
            rows.append(X)
            cols.append(min(max(q, 0), size - 1))
            values.append(max(0.0, 1 - abs(src - q)) if bilinear else cubic(src - q))
    out = torch.zeros((size * scale, size), dtype=torch.float64, device="cuda")
    return out.index_put_((torch.tensor(rows, device="cuda"), torch.tensor(cols, device="cuda")), torch.tensor(values, dtype=torch.float64, device="cuda"), accumulate=True)


def _exact_grad(state):
    """By differentiating the regression's own definition, frame by frame and tap by tap."""
    case = state["case"]
    n, c, h, w, r, D, k, s = (case[x] for x in ("n", "c", "h", "w", "scale", "D", "k", "s"))
    H, W, p, mode = h * r, w * r, (k - 1) // 2, case["mode"]
    My, Mx = _matrix(h, r, case["bilinear"]), _matrix(w, r, case["bilinear"])
    dict_ = state["dict"].double().requires_grad_()
    gamma = state["gamma"].double().requires_grad_() if mode == "global" else None
    g_dict, g_gamma, g_coef = torch.zeros_like(dict_), None if gamma is None else torch.zeros_like(gamma), []
    for f in range(n):
        u = torch.nn.functional.pad(My @ state["lr"][f].double() @ Mx.t(), (p, p, p, p), mode="replicate")
        coef = state["coef"][f].double().requires_grad_()
        if mode == "dense":
            phi, atoms = coef, dict_
        elif mode == "global":
            at = state["idx"].long()
            phi, atoms = coef[at] * gamma.view(-1, 1, 1), dict_[at]
        elif mode == "compact":
            phi, atoms = torch.zeros((D, H, W), dtype=torch.float64, device="cuda").scatter(0, state["idx"][f].long(), coef), dict_
        else:
            phi, atoms = coef * torch.zeros_like(coef).scatter(0, state["idx"][f].long(), 1.0), dict_
        filters = (atoms.t() @ phi.flatten(1)).view(k * k, H, W)
        G = state["grad_out"][f].double()
        d_filters = torch.stack([(u[:, a:a + H, b:b + W] * G).sum(0) for a in range(k) for b in range(k)])
        wrt = [coef, dict_] + ([gamma] if gamma is not None else [])
        got = torch.autograd.grad(filters, wrt, d_filters)
        g_coef.append(got[0])
        g_dict = g_dict + got[1]
        if gamma is not None:
            g_gamma = g_gamma + got[2]
        del filters, d_filters, phi, coef, got
    both = torch.stack(g_coef), g_dict.detach()
    return both if mode == "dense" else (*both, g_gamma)


def _exact_balance(state):
    """By differentiating the loss."""
    case, idx = state["case"], state["idx"]
    n, H, W, D, s = (case[x] for x in ("n", "H", "W", "D", "s"))
    on = torch.ones((n, H, W), dtype=torch.float64, device="cuda") if state["mask"] is None else state["mask"].double()
    counts = torch.stack([torch.bincount((idx[f].long() + 1)[(on[f] > 0).expand(s, H, W)], minlength=D + 1)[1:] for f in range(n)])
    valid = on.sum((1, 2))
    slope = counts.double() / s / (n * valid.clamp(min=1) ** 2).view(n, 1) if case["per_frame"] else (counts.sum(0) / s / valid.sum().clamp(min=1) ** 2).expand(n, D)
    loss, shares, grads = 0.0, [], []
    for f in range(n):
        coef = state["coef"][f].double().requires_grad_()
        total = coef.abs().sum(0)
        empty = total == 0
        p = torch.where(empty, torch.full_like(coef, 1.0 / D), coef.abs() / torch.where(empty, torch.ones_like(total), total)) * on[f]
        if case["per_frame"]:
            part = D / n * (counts[f] / (s * valid[f].clamp(min=1)) * p.sum((1, 2)) / valid[f].clamp(min=1)).sum()
        else:
            part = D * (counts.sum(0) / (s * valid.sum().clamp(min=1)) * p.sum((1, 2)) / valid.sum().clamp(min=1)).sum()
        grads.append(torch.autograd.grad(part, coef)[0] * state["weight"])
        loss = loss + part.detach()
        shares.append((p.sum((1, 2)) / valid[f].clamp(min=1)).detach())
    grad = torch.stack(grads)
    if case["add"]:
        grad += state["grad"]
    return loss.view(1), counts.int(), torch.stack(shares), D * slope, grad


def _exact_adamw(state):
    o, t = {k: float(v) for k, v in state["opts"].items()}, state["step"]
    eight = state["case"]["bits"] == 8
    unpack = lambda x, scale: x.double() * scale.double().repeat_interleave(QUANT_BLOCK) if eight else x.double()  # noqa: E731
    m, v = unpack(state["m"], state.get("m_scale")), unpack(state["v"], state.get("v_scale"))
    v = v.square() if eight else v
    g = state["grad"].double() * o["grad_scale"]
    m.mul_(o["beta1"]).add_(g, alpha=1 - o["beta1"])
    v.mul_(o["beta2"]).addcmul_(g, g, value=1 - o["beta2"])
    m_hat, v_hat = m / (1 - o["beta1"] ** t), v / (1 - o["beta2"] ** t)
    p = state["param"].double()
    p = p - o["lr"] * (m_hat / (v_hat.sqrt() + o["eps"]) + o["weight_decay"] * p)
    if not eight:
        return [p, m, v]
    scales = [x.abs().view(-1, QUANT_BLOCK).amax(1) / F8_MAX for x in (m, v.sqrt())]
    return [p, None, None] + scales                            # the 8-bit values are held to the plain form's


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        total, size = sum(_adamw_sizes(case)), {"f32": 4, "f16": 2, "bf16": 2}
        state = 16 if case["bits"] == 32 else 4 + 16 / QUANT_BLOCK
        return {"bytes": total * (2 * size[case["param"]] + size[case["grad"]] + state), "flops": 14 * total}
    e, D, s = {"f32": 4, "f16": 2}[case["dtype"]], case["D"], case["s"]
    if case["op"] == "balance":
        px = case["n"] * case["H"] * case["W"]
        # coefficients once for the loss and once for its gradient (which needs the whole loss first), the gradient written (and read)
        return {"bytes": px * (e * D * (4 if case["add"] else 3) + s + 2 * case["masked"]), "flops": px * D * 8}
    px, kk = case["n"] * case["h"] * case["w"] * case["scale"] ** 2, case["k"] ** 2
    used = D if case["mode"] == "dense" else s                 # atoms whose products count at a pixel
    written = s if case["mode"] == "compact" else D
    per_pixel = e * (used + written) + (s if case["mode"] in ("listed", "compact") else 0) + 4 * case["c"] * (1 + 1 / case["scale"] ** 2)
    return {"bytes": px * per_pixel + 8 * D * kk, "flops": px * (4 * used * kk + 2 * case["c"] * kk)}
