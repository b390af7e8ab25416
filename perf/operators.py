"""Adapters beside a shared compressed projection, and the AdamW step that trains them, as cases that can be timed and compared.

``own`` chooses what ``run`` computes: the calls of this framework, or the same operators in elementary torch operations.

project    z[t] = s_a (x[t] A_a^T), y[t] = x[t] W^T + z[t] B_a^T, where a is the adapter of token t (-1: none, z = 0)
backward   dz[t] = s_a dy[t] B_a, dx[t] = dy[t] W + dz[t] A_a, dA_a = sum of dz[t]^T x[t], dB_a = sum of dy[t]^T z[t] over a's tokens
adamw      one AdamW update of a list of tensors, with the L-C penalty folded in or without, states in 32 bits or in e4m3 codes with
           a scale for every 256 elements, the codes rounded to nearest or by random bits that a seed gives

All tensors of one kind of an AdamW case are views of one buffer, each starting at a multiple of 256 elements with zeros in between.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
BLOCK = 256                                # elements of a tensor that share the scale of an 8-bit state
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.999, 1e-8, 0.01, 1e-3
MU = 1e-3


# ---- the cases --------------------------------------------------------------------------------------------------

def _vgg19():
    out, cin = [], 3
    for c in (64, 64, 128, 128, 256, 256, 256, 256, 512, 512, 512, 512, 512, 512, 512, 512):
        out.append((c, cin, 3, 3))
        cin = c
    return out + [(10, 512)]


def _transformer_base():
    encoder = [(512, 512)] * 4 + [(2048, 512), (512, 2048)]
    decoder = [(512, 512)] * 8 + [(2048, 512), (512, 2048)]
    return encoder * 6 + decoder * 6


MODELS = {"vgg19": _vgg19, "transformer": _transformer_base}


def _shapes(case):
    text = case["shapes"]
    if text in MODELS:
        return MODELS[text]()
    out = []
    for part in text.split(","):
        count, _, dims = part.rpartition("*")
        out += [tuple(int(d) for d in dims.split("x"))] * int(count or 1)
    return out


def listed():
    return [
        # one new token of one request through a Transformer-base's wide layer: the smallest call
        {"name": "project-1", "op": "project", "type": "bf16", "tokens": 1, "requests": 1, "n_in": 512, "n_out": 2048, "adapters": 16, "rank": 8, "ragged": False},
        # one new token of each of 64 requests, with adapters of their own: a serving step of a large model's layer
        {"name": "project-64-requests", "op": "project", "type": "bf16", "tokens": 64, "requests": 64, "n_in": 4608, "n_out": 4096, "adapters": 64, "rank": 16, "ragged": False},
        # prompts of nine requests, some without an adapter, ranks of all kinds, through an LSTM's gates (rows that are not 16-byte aligned)
        {"name": "project-prompts-odd", "op": "project", "type": "f16", "tokens": 1333, "requests": 9, "n_in": 650, "n_out": 2600, "adapters": 12, "rank": 24, "ragged": True},
        # a training batch of a large model's layer, eight adapters trained at once
        {"name": "project-train", "op": "project", "type": "bf16", "tokens": 8192, "requests": 16, "n_in": 4608, "n_out": 4096, "adapters": 8, "rank": 16, "ragged": False},
        # gradients of a small batch of the Transformer-base layer
        {"name": "backward-128", "op": "backward", "type": "bf16", "tokens": 128, "requests": 4, "n_in": 512, "n_out": 2048, "adapters": 4, "rank": 8, "ragged": False},
        # gradients of ragged prompts through the LSTM's gates
        {"name": "backward-odd", "op": "backward", "type": "f16", "tokens": 1333, "requests": 9, "n_in": 650, "n_out": 2600, "adapters": 5, "rank": 24, "ragged": True},
        # gradients of the training batch
        {"name": "backward-train", "op": "backward", "type": "bf16", "tokens": 8192, "requests": 16, "n_in": 4608, "n_out": 4096, "adapters": 8, "rank": 16, "ragged": False},
        # the adapters of one small layer: the smallest update
        {"name": "adamw-adapters", "op": "adamw", "shapes": "4*8x512,4*2048x8", "states": 32, "grads": "f32", "penalty": False, "codes": "bf16", "stochastic": False},
        # the learning step of the VGG-19 with the L-C penalty
        {"name": "adamw-vgg19-lc", "op": "adamw", "shapes": "vgg19", "states": 32, "grads": "f32", "penalty": True, "codes": "none", "stochastic": False},
        # a Transformer-base with gradients and forward weights in 16 bits and states in 8, rounded by random bits
        {"name": "adamw-transformer-8bit", "op": "adamw", "shapes": "transformer", "states": 8, "grads": "bf16", "penalty": False, "codes": "bf16", "stochastic": True},
        # matrices that nothing divides, states in 8 bits with the penalty
        {"name": "adamw-odd-8bit", "op": "adamw", "shapes": "8*2600x651,5*333x331,3*77", "states": 8, "grads": "f16", "penalty": True, "codes": "f16", "stochastic": False},
        # 604 million weights of a large model with states in 32 bits
        {"name": "adamw-large", "op": "adamw", "shapes": "32*4096x4608", "states": 32, "grads": "f32", "penalty": True, "codes": "bf16", "stochastic": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, hi):
    """A number of channels: odd ones, multiples of 2, 8 and 64."""
    n = _log_int(rng, 64, hi)
    unit = rng.choice((1, 2, 8, 64, 64))
    return max(unit, n // unit * unit)


def draw(rng):
    op = rng.choice(("project", "project", "backward", "adamw", "adamw"))
    if op == "adamw":
        elems, n = _log_int(rng, 1 << 12, 1 << 28), _log_int(rng, 1, 200)
        rows = max(1, int(math.sqrt(elems / n) * math.exp(rng.uniform(-0.8, 0.8))))
        cols = max(1, elems // n // rows)
        return {"op": op, "shapes": "%d*%dx%d,%d*%d" % (n, rows, cols, rng.randint(1, 4), rng.randint(1, 700)), "states": rng.choice((8, 32)),
                "grads": rng.choice(("f32", "bf16", "f16")), "penalty": rng.random() < 0.5, "codes": rng.choice(("none", "bf16", "f16")), "stochastic": rng.random() < 0.5}
    tokens = _log_int(rng, 1, 8192)
    adapters = rng.randint(1, 24)
    return {"op": op, "type": rng.choice(("bf16", "f16")), "tokens": tokens, "requests": min(tokens, _log_int(rng, 1, 256)),
            "n_in": _side(rng, 4608), "n_out": _side(rng, 4096), "adapters": adapters, "rank": rng.randint(1, 64), "ragged": rng.random() < 0.5}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _host_choices(case, seed):
    """Ranks of the adapters, their scales, and the adapter of every token: requests of random lengths, one in nine without an adapter."""
    g = torch.Generator().manual_seed(seed * 2 + 1)
    n, r = case["adapters"], case["rank"]
    own_ranks = torch.Generator().manual_seed(n * 1000 + r)               # the adapters that a program holds, whatever the batch
    ranks = torch.randint(1, r + 1, (n,), generator=own_ranks) if case["ragged"] else torch.full((n,), r)
    scales = 2.0 ** torch.randint(-1, 2, (n,), generator=g).double()
    R, T = case["requests"], case["tokens"]
    if R == T:
        owner = torch.arange(T)
    else:
        cuts = torch.randperm(T - 1, generator=g)[: R - 1].sort().values + 1
        owner = torch.bucketize(torch.arange(T), cuts, right=True)
    adapter = torch.arange(R) % n if R <= n else torch.randint(0, n, (R,), generator=g)
    adapter = torch.where(torch.rand(R, generator=g) < 1 / 9, torch.full_like(adapter, -1), adapter)
    return ranks.tolist(), [float(s) for s in scales], adapter[owner].to(torch.int32)


def _prepare_adapters(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    t, T, K, N = TYPES[case["type"]], case["tokens"], case["n_in"], case["n_out"]

    def normal(std, *shape):
        return (torch.randn(*shape, device=DEVICE, generator=g) * std).to(t)

    ranks, scales, ids = _host_choices(case, seed)
    s = {"op": case["op"], "ranks": ranks, "max_rank": case["rank"], "type": t, "ids": ids.to(DEVICE)}
    w = normal(0.02, N, K)
    s["w"] = torch.where(torch.rand(N, K, device=DEVICE, generator=g) < 0.5, w, torch.zeros_like(w))      # pruned to one half
    s["x"] = normal(1.0, T, K)
    s["a"] = [normal(1 / math.sqrt(K), r, K) for r in ranks]
    s["b"] = [normal(0.02, N, r) for r in ranks]
    owner = torch.cat([torch.full((r,), i) for i, r in enumerate(ranks)])
    s["owner"] = owner.to(DEVICE)                                        # the adapter that a row of all A's together belongs to
    s["row0"] = torch.tensor([sum(ranks[:i]) for i in range(len(ranks))], device=DEVICE)
    s["rank_of"] = torch.tensor(ranks, device=DEVICE)
    s["scale_of"] = torch.tensor(scales, device=DEVICE, dtype=torch.float64)
    s["scales"] = scales
    grads = None
    if case["op"] == "backward":
        s["dy"] = normal(0.01, T, N)
        z = torch.randn(T, case["rank"], device=DEVICE, generator=g)     # as the forward pass kept it: zero where there is no row of A
        rank_of_token = torch.where(s["ids"] < 0, torch.zeros_like(s["ids"]), s["rank_of"][s["ids"].clamp(min=0).long()].to(torch.int32))
        s["z"] = torch.where(torch.arange(case["rank"], device=DEVICE)[None] < rank_of_token[:, None], z, torch.zeros_like(z)).to(t)
        grads = [(torch.empty(r, K, device=DEVICE), torch.empty(N, r, device=DEVICE)) for r in ranks]
        s["dx"] = torch.empty(T, K, device=DEVICE, dtype=t)
    else:
        s["y"] = torch.empty(T, N, device=DEVICE, dtype=t)
        s["z"] = torch.empty(T, case["rank"], device=DEVICE, dtype=t)
    s["grads"] = grads
    if own:
        import paper_1911_02497_amd as P
        s["table"] = P.adapter_table(list(zip(s["a"], s["b"], scales)), grads=grads)
        s["workspace"] = P.adapter_workspace(s["table"], T, backward=grads is not None)
    return s


def _prepare_adamw(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    shapes = _shapes(case)
    sizes = [math.prod(sh) for sh in shapes]
    starts, n = [], 0
    for size in sizes:
        starts.append(n)
        n += -(-size // BLOCK) * BLOCK
    begin = torch.tensor(starts, device=DEVICE).div(BLOCK, rounding_mode="floor")
    ends = torch.tensor([a + b for a, b in zip(starts, sizes)], device=DEVICE)
    inside = torch.arange(n, device=DEVICE) < ends[torch.searchsorted(begin, torch.arange(n // BLOCK, device=DEVICE), right=True) - 1].repeat_interleave(BLOCK)

    def normal(std, t=torch.float32):
        return (torch.randn(n, device=DEVICE, generator=g) * std).mul_(inside).to(t)

    def views(flat):
        return [flat[a:a + size].view(sh) for a, size, sh in zip(starts, sizes, shapes)]

    s = {"op": "adamw", "states": case["states"], "stochastic": case["stochastic"], "n": n, "seed": seed * 0x9E3779B97F4A7C15 % (1 << 64), "step": 1 + seed % 1000}
    s["w"] = normal(0.02)
    s["grad"] = normal(1e-3, TYPES[case["grads"]])
    s["theta"], s["lam"] = (torch.where(s["w"].abs() > 0.03, s["w"], torch.zeros_like(s["w"])), normal(1e-4)) if case["penalty"] else (None, None)
    s["codes"] = None if case["codes"] == "none" else torch.zeros(n, device=DEVICE, dtype=TYPES[case["codes"]])
    if case["states"] == 32:
        s["m"], s["v"] = normal(3e-4), normal(1e-3).square_()
    else:
        for k, std in (("m", 3e-4), ("r", 1e-3)):
            x = normal(std)
            x = x.abs_() if k == "r" else x
            scale = x.view(-1, BLOCK).abs().amax(1) / 448
            s[k] = (x.view(-1, BLOCK) / scale[:, None].clamp(min=1e-30)).clamp(-448, 448).view(-1).to(torch.float8_e4m3fn).view(torch.uint8)
            s[k + "_scale"] = scale
            del x
    if own:
        import paper_1911_02497_amd as P

        def scales(flat):
            return [flat[a // BLOCK:-(-(a + size) // BLOCK)] for a, size in zip(starts, sizes)]

        more = {}
        if case["penalty"]:
            more.update(theta=views(s["theta"]), lambdas=views(s["lam"]))
        if s["codes"] is not None:
            more.update(codes=views(s["codes"]))
        if case["states"] == 8:
            more.update(exp_avg_scale=scales(s["m_scale"]), exp_avg_sq_scale=scales(s["r_scale"]))
        s["table"] = P.adamw_table(views(s["w"]), views(s["grad"]), views(s["m"]), views(s["v" if case["states"] == 32 else "r"]), **more)
    return s


def prepare(case, seed):
    return _prepare_adamw(case, seed) if case["op"] == "adamw" else _prepare_adapters(case, seed)


# ---- one pass ---------------------------------------------------------------------------------------------------

def _own(s):
    import paper_1911_02497_amd as P
    if s["op"] == "project":
        P.condensa_adapter_project(s["x"], s["w"], s["table"], s["ids"], y=s["y"], z=s["z"], workspace=s["workspace"])
        return {"y": s["y"], "z": s["z"]}
    if s["op"] == "backward":
        P.condensa_adapter_project_backward(s["dy"], s["x"], s["w"], s["table"], s["ids"], s["z"], dx=s["dx"], workspace=s["workspace"])
        return {"dx": s["dx"], "da": [a for a, _ in s["grads"]], "db": [b for _, b in s["grads"]]}
    P.condensa_lc_adamw_step(s["table"], LR, s["step"], betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY, mu=MU,
                             seed=s["seed"] if s["stochastic"] else None)
    return _states(s)


def _states(s):
    out = {"w": s["w"]} if s["codes"] is None else {"w": s["w"], "codes": s["codes"]}
    if s["states"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    return {**out, "m": s["m"].view(torch.float8_e4m3fn), "r": s["r"].view(torch.float8_e4m3fn), "m_scale": s["m_scale"], "r_scale": s["r_scale"]}


def _mine(s):
    """1 where a row of all A's together is of the token's adapter, times the adapter's scale."""
    return (s["ids"][:, None] == s["owner"][None]).float() * s["scale_of"].float()[s["owner"]][None]


def _own_rows(s, zfull):
    """[T, max_rank]: the columns of the token's own adapter."""
    a = s["ids"].long()
    j = torch.arange(s["max_rank"], device=DEVICE)[None]
    there = (a[:, None] >= 0) & (j < s["rank_of"][a.clamp(min=0)][:, None])
    at = (s["row0"][a.clamp(min=0)][:, None] + j).clamp(max=zfull.shape[1] - 1)
    return torch.where(there, zfull.gather(1, at), torch.zeros((), device=DEVICE, dtype=zfull.dtype))


def _plain_project(s):
    x, a, b = s["x"].float(), torch.cat(s["a"]).float(), torch.cat(s["b"], 1).float()
    z = (x @ a.t()) * _mine(s)
    return {"y": (x @ s["w"].float().t() + z @ b.t()).to(s["type"]), "z": _own_rows(s, z).to(s["type"])}


def _plain_backward(s):
    dy, x, a, b = s["dy"].float(), s["x"].float(), torch.cat(s["a"]).float(), torch.cat(s["b"], 1).float()
    mine = _mine(s)
    dz = (dy @ b) * mine
    dx = (dy @ s["w"].float() + dz @ a).to(s["type"])
    first = torch.arange(s["owner"].numel(), device=DEVICE) - s["row0"][s["owner"]]          # a row of all A's together in its own A
    z = s["z"].float()[:, first] * (mine != 0)
    da, db = dz.t() @ x, dy.t() @ z
    return {"dx": dx, "da": list(torch.split(da, s["ranks"])), "db": [t.contiguous() for t in torch.split(db, s["ranks"], 1)]}


def _mix(x, mul):
    return (x * mul) & 0xFFFFFFFF


def _noise(s):
    """32 random bits for every element: the integer hash "lowbias32" (C. Wellons) of its position, with halves of the seed mixed in before and between."""
    p = torch.arange(s["n"], device=DEVICE)
    h = (p & 0xFFFFFFFF) ^ _mix(p >> 32, 0x9E3779B9) ^ (s["seed"] & 0xFFFFFFFF)
    h = _mix(h ^ (h >> 16), 0x7FEB352D)
    h = ((h ^ (h >> 15)) + (s["seed"] >> 32)) & 0xFFFFFFFF
    h = _mix(h, 0x846CA68B)
    return h ^ (h >> 16)


def _encode(x, noise, at_least_one):
    """e4m3 codes of x in blocks of 256 and their scales; `noise`: 16 random bits that decide between the two neighbours, or None for the nearest."""
    block = x.view(-1, BLOCK)
    size = block.abs()
    top = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax(1, keepdim=True)
    kept = top >= 2.0 ** -100
    top = torch.where(kept, top, torch.ones_like(top))
    y = (size * torch.where(kept, 448 / top, torch.zeros_like(top))).view(-1)
    if noise is None:
        code = y.clamp(max=448).to(torch.float8_e4m3fn).view(torch.uint8).int()
    else:
        bits = y.view(torch.int32)
        normal = ((bits.clamp(max=0x7F7FFFFF) + (noise << 4)) >> 20) - (120 << 3)
        small = ((y.clamp(max=1) * 2.0 ** 29).int() + (noise << 4)) >> 20
        code = torch.where(y >= 2.0 ** -6, normal, small)
    code = code.clamp(max=0x7E)
    if at_least_one:
        code = torch.where((x > 0) & kept.expand(-1, BLOCK).reshape(-1), code.clamp(min=1), code)
    code = torch.where(torch.isnan(x), torch.full_like(code, 0x7F), code)
    code = code | torch.where(torch.signbit(x), 128, 0).int()
    return code.to(torch.uint8), torch.where(kept, top / 448, torch.zeros_like(top)).view(-1)


def _f32(x):
    return torch.tensor(x, dtype=torch.float32).item()


def _plain_adamw(s):
    t = s["step"]
    step_size, correct = _f32(LR / (1 - BETA1 ** t)), _f32(1 / math.sqrt(1 - BETA2 ** t))
    g = s["grad"].float()
    if s["theta"] is not None:
        g = (g + (s["w"] - s["theta"]) * _f32(MU)) - s["lam"]
    if s["states"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["r"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["r_scale"][:, None]).view(-1).square()
    m = m * _f32(BETA1) + g * _f32(1 - BETA1)
    v = v * _f32(BETA2) + (g * g) * _f32(1 - BETA2)
    r = v.sqrt()
    s["w"].copy_(s["w"] * _f32(1 - LR * DECAY) - (m / (r * correct + _f32(EPS))) * step_size)
    if s["codes"] is not None:
        s["codes"].copy_(s["w"])
    if s["states"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        noise = _noise(s).int() if s["stochastic"] else None
        for k, x, bits in (("m", m, None if noise is None else noise & 0xFFFF), ("r", r, None if noise is None else (noise >> 16) & 0xFFFF)):
            code, scale = _encode(x, bits, k == "r")
            s[k].copy_(code)
            s[k + "_scale"].copy_(scale)
    return _states(s)


def run(state):
    if own:
        return _own(state)
    return {"project": _plain_project, "backward": _plain_backward, "adamw": _plain_adamw}[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n = sum(math.prod(sh) for sh in _shapes(case))
        state = 16 if case["states"] == 32 else 4 + 16 / BLOCK
        per = 8 + state + (4 if case["grads"] == "f32" else 2) + (8 if case["penalty"] else 0) + (0 if case["codes"] == "none" else 2)
        return {"bytes": n * per, "flops": n * (14 + (3 if case["penalty"] else 0))}
    T, K, N, n = case["tokens"], case["n_in"], case["n_out"], case["adapters"]
    r = (case["rank"] + 1) / 2 if case["ragged"] else case["rank"]
    used = min(n, case["requests"]) * r
    if case["op"] == "project":
        return {"bytes": 2 * (T * K + N * K + used * (K + N) + T * N + T * r), "flops": 2 * T * N * K + 2 * T * r * (K + N)}
    return {"bytes": 2 * (2 * T * K + T * N + N * K + used * (K + N) + T * r) + 4 * n * r * (K + N), "flops": 2 * T * N * K + 4 * T * r * (K + N)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _exact_adapters(s):
    ids = s["ids"].tolist()
    x, w = s["x"].double(), s["w"].double()
    rows = {a: torch.tensor([t for t, i in enumerate(ids) if i == a], device=DEVICE, dtype=torch.long) for a in range(len(s["ranks"]))}
    if s["op"] == "project":
        y = x.mm(w.t())
        z = torch.zeros(len(ids), s["max_rank"], device=DEVICE, dtype=torch.float64)
        for a, at in rows.items():
            if at.numel():
                zs = x[at].mm(s["a"][a].double().t()) * s["scales"][a]
                z[at, :s["ranks"][a]] = zs
                y[at] += zs.mm(s["b"][a].double().t())
        return {"y": y, "z": z}
    dy = s["dy"].double()
    dx, da, db = dy.mm(w), [], []
    for a, at in rows.items():
        r = s["ranks"][a]
        dz = dy[at].mm(s["b"][a].double()) * s["scales"][a]
        dx[at] += dz.mm(s["a"][a].double())
        da.append(dz.t().contiguous().mm(x[at]))
        db.append(dy[at].t().contiguous().mm(s["z"][at, :r].double()))
    return {"dx": dx, "da": da, "db": db}


def _exact_codes(x, noise, at_least_one):
    """Values of the e4m3 grid next to x / scale: multiples of 2^(e-3), e the exponent of x / scale and at least -6; and the scales."""
    finite = torch.nan_to_num(x.abs(), nan=0.0, posinf=0.0).reshape(-1, BLOCK)
    scale = finite.amax(1) / 448
    scale = torch.where(scale * 448 < 2.0 ** -100, torch.zeros_like(scale), scale)
    q = torch.where(scale[:, None] > 0, x.reshape(-1, BLOCK).abs() / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None], torch.zeros_like(finite)).reshape(-1)
    step = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -6))) - 3)
    units = q / step
    units = torch.round(units) if noise is None else torch.floor(units + noise.double() / 65536)
    q = (units * step).clamp(max=448)
    if at_least_one:
        q = torch.where((x > 0) & (scale.repeat_interleave(BLOCK) > 0), q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, x), scale


def _exact_adamw(s):
    d = {k: v.double() for k, v in s.items() if k in ("w", "grad", "theta", "lam", "v") and v is not None}
    t, g = s["step"], d["grad"]
    if "theta" in d:
        g = g + MU * (d["w"] - d["theta"]) - d["lam"]
    if s["states"] == 32:
        m, v = s["m"].double(), d["v"]
    else:
        m = s["m"].view(torch.float8_e4m3fn).double() * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (s["r"].view(torch.float8_e4m3fn).double() * s["r_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    w = d["w"] - LR * DECAY * d["w"] - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"w": w} if s["codes"] is None else {"w": w, "codes": w}
    if s["states"] == 32:
        return {**out, "m": m, "v": v}
    h = None
    if s["stochastic"]:
        low, high = s["seed"] % (1 << 32), s["seed"] >> 32
        p = torch.arange(s["n"], device=DEVICE)
        h = (p % (1 << 32)) ^ ((p // (1 << 32) * 0x9E3779B9) % (1 << 32)) ^ low
        h = ((h ^ (h >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
        h = (((h ^ (h >> 15)) + high) * 0x846CA68B) & 0xFFFFFFFF
        h = h ^ (h >> 16)
    (mq, ms), (rq, rs) = _exact_codes(m, None if h is None else h & 0xFFFF, False), _exact_codes(torch.sqrt(v), None if h is None else h >> 16, True)
    return {**out, "m": mq, "r": rq, "m_scale": ms, "r_scale": rs}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_adapters(s)
