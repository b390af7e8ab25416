"""Products with matrices held in 8 bits, a scale for each block of 128, and the norms that feed them, as cases that can be timed and compared.

``own`` chooses what ``run`` computes: the calls of this framework, or the same operators in elementary torch operations.

codec      e4m3 codes of a matrix and their scales, one for every 128 columns of a row or of 128 rows, and the values that they stand for
norm       h = x + residual, rounded to the 16-bit type, y = h / sqrt(mean h^2 + eps) * weight, in 16 bits or in codes with a scale for 128 columns
norm-back  from dy and what reaches h elsewhere: the gradient of h (in 16 bits, and in codes) and of the weight
project    y = x W^T, x in codes with a scale for 128 columns of a token, W in codes with a scale for 128 x 128
back       dx = dy W, the same W, dy in codes with a scale for 128 columns of a token

Scales are (largest finite magnitude of the block) / 448; codes are rounded to the nearest, ties to even.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
BLOCK = 128                                # columns (and rows, of a weight matrix) that share a scale
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- the cases --------------------------------------------------------------------------------------------------

def listed():
    return [
        # one new token of one request in front of a Transformer-base's layer: the smallest norm
        {"name": "norm-1", "op": "norm", "type": "bf16", "tokens": 1, "width": 512, "residual": True, "wide": False, "codes": True, "weight": "bf16"},
        # ragged prompts in front of an LSTM's gates (rows that are not 16-byte aligned), beside a layer that wants 16 bits
        {"name": "norm-odd", "op": "norm", "type": "f16", "tokens": 1333, "width": 650, "residual": True, "wide": True, "codes": True, "weight": "f32"},
        # a training batch in front of a large model's layer
        {"name": "norm-train", "op": "norm", "type": "bf16", "tokens": 8192, "width": 4608, "residual": True, "wide": False, "codes": True, "weight": "bf16"},
        # its gradients for the ragged prompts
        {"name": "norm-back-odd", "op": "norm-back", "type": "f16", "tokens": 1333, "width": 650, "residual": False, "codes": False, "weight": "f32"},
        # and for the training batch, in 16 bits for the residual and in codes for the layer before it
        {"name": "norm-back-train", "op": "norm-back", "type": "bf16", "tokens": 8192, "width": 4608, "residual": True, "codes": True, "weight": "bf16"},
        # what passes from the LSTM's gates to a product, and back
        {"name": "codec-rows-odd", "op": "codec", "type": "f16", "rows": 1333, "cols": 2600, "block_rows": 1},
        # the weights of a large model's layer as the compression step left them
        {"name": "codec-weights", "op": "codec", "type": "f32", "rows": 4096, "cols": 4608, "block_rows": 128},
        # one new token through a Transformer-base's wide layer: the smallest product
        {"name": "project-1", "op": "project", "type": "bf16", "tokens": 1, "n_in": 512, "n_out": 2048, "contiguous": False},
        # one new token of each of 64 requests: a serving step of a large model's layer
        {"name": "project-64", "op": "project", "type": "bf16", "tokens": 64, "n_in": 4608, "n_out": 4096, "contiguous": False},
        # a training batch of a large model's layer
        {"name": "project-train", "op": "project", "type": "bf16", "tokens": 8192, "n_in": 4608, "n_out": 4096, "contiguous": False},
        # gradients of ragged prompts through the LSTM's gates
        {"name": "back-odd", "op": "back", "type": "f16", "tokens": 1333, "n_in": 650, "n_out": 2600, "contiguous": False},
        # gradients of the training batch
        {"name": "back-train", "op": "back", "type": "bf16", "tokens": 8192, "n_in": 4608, "n_out": 4096, "contiguous": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, lo, hi):
    """A number of channels: odd ones, multiples of 2, 16 and 128."""
    n = _log_int(rng, lo, hi)
    unit = rng.choice((1, 2, 16, 128, 128))
    return max(unit, n // unit * unit)


def draw(rng):
    op = rng.choice(("norm", "norm-back", "codec", "project", "project", "back"))
    kind = rng.choice(("bf16", "f16"))
    if op == "codec":
        rows = _log_int(rng, 1, 4096)
        return {"op": op, "type": rng.choice(("f32", kind)), "rows": rows, "cols": _side(rng, 64, 4608), "block_rows": rng.choice((1, 128))}
    if op in ("norm", "norm-back"):
        width = _side(rng, 64, 16384)
        case = {"op": op, "type": kind, "tokens": _log_int(rng, 1, min(8192, 8192 * 4608 // width)), "width": width, "residual": rng.random() < 0.7}
        codes = rng.random() < 0.7
        if op == "norm":
            case["wide"] = not codes or rng.random() < 0.3
        return {**case, "codes": codes, "weight": rng.choice(("f32", kind))}
    return {"op": op, "type": kind, "tokens": _log_int(rng, 1, 8192), "n_in": _side(rng, 64, 4608), "n_out": _side(rng, 64, 4096), "contiguous": rng.random() < 0.2}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _blocks(n):
    return -(-n // BLOCK)


def _empty_codes(rows, cols, block_rows=1, contiguous=False):
    """Codes in rows that begin at multiples of 128 bytes, or one behind the other, and their scales."""
    q = torch.zeros(rows, cols if contiguous else _blocks(cols) * BLOCK, dtype=torch.uint8, device=DEVICE)[:, :cols]
    return q, torch.empty(-(-rows // block_rows), _blocks(cols), device=DEVICE)


def _made_codes(x, block_rows, contiguous):
    q, scale = _empty_codes(*x.shape, block_rows, contiguous)
    codes, s = _encode(x, block_rows)
    q.copy_(codes.view(torch.uint8))
    scale.copy_(s)
    return q, scale


def _activations(case, rows, cols, normal, g):
    """Channels of different sizes, some of them many times the others'."""
    size = torch.exp(0.5 * torch.randn(cols, device=DEVICE, generator=g))
    size = torch.where(torch.rand(cols, device=DEVICE, generator=g) < 0.01, size * 20, size)
    return normal(1.0, rows, cols) * size


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(std, *shape):
        return torch.randn(*shape, device=DEVICE, generator=g) * std

    s = {"op": case["op"], "type": t}
    if case["op"] == "codec":
        rows, cols = case["rows"], case["cols"]
        x = normal(0.02, rows, cols) if case["block_rows"] > 1 else _activations(case, rows, cols, normal, g)
        if case["block_rows"] > 1:                                       # pruned to one half
            x = torch.where(torch.rand(rows, cols, device=DEVICE, generator=g) < 0.5, x, torch.zeros_like(x))
        s["x"], s["block_rows"] = x.to(t), case["block_rows"]
        s["q"], s["scale"] = _empty_codes(rows, cols, case["block_rows"])
        s["back"] = torch.empty(rows, cols, device=DEVICE, dtype=t)
    elif case["op"] in ("norm", "norm-back"):
        T, n = case["tokens"], case["width"]
        s["weight"] = (1 + normal(0.2, n)).to(TYPES[case["weight"]])
        s["q"], s["scale"] = _empty_codes(T, n) if case["codes"] else (None, None)
        if case["op"] == "norm":
            s["x"] = normal(0.5, T, n).to(t)
            s["residual"] = _activations(case, T, n, normal, g).to(t) if case["residual"] else None
            s["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
            s["y"] = torch.empty_like(s["x"]) if case["wide"] else None
        else:
            s["h"], s["dy"] = _activations(case, T, n, normal, g).to(t), normal(0.01, T, n).to(t)
            s["dsum"] = normal(0.01, T, n).to(t) if case["residual"] else None
            s["dx"], s["dweight"] = torch.empty_like(s["h"]), torch.empty(n, device=DEVICE)
    else:
        T, K, N = case["tokens"], case["n_in"], case["n_out"]
        w = normal(0.02, N, K)
        w = torch.where(torch.rand(N, K, device=DEVICE, generator=g) < 0.5, w, torch.zeros_like(w))       # pruned to one half
        s["w"], s["w_scale"] = _made_codes(w, BLOCK, case["contiguous"])
        x = _activations(case, T, K, normal, g) if case["op"] == "project" else normal(0.01, T, N)
        s["x"], s["x_scale"] = _made_codes(x, 1, case["contiguous"])
        s["y"] = torch.empty(T, N if case["op"] == "project" else K, device=DEVICE, dtype=t)
    if own:
        import paper_1911_02497_amd as P
        if "w" in s:
            s["W"], s["X"] = P.Fp8Matrix(s["w"], s["w_scale"], BLOCK), P.Fp8Matrix(s["x"], s["x_scale"], 1)
            s["workspace"] = P.project_fp8_workspace(s["W"], case["tokens"], backward=case["op"] == "back")
        elif s["q"] is not None:
            s["Q"] = P.Fp8Matrix(s["q"], s["scale"], s.get("block_rows", 1))
        if case["op"] == "norm-back":
            s["workspace"] = P.rms_norm_workspace(case["tokens"], case["width"], DEVICE)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------

def _own(s):
    import paper_1911_02497_amd as P
    if s["op"] == "codec":
        P.condensa_quantize_fp8_blocks(s["x"], out=s["Q"])
        P.condensa_dequantize_fp8_blocks(s["Q"], out=s["back"])
        return {"codes": s["q"].view(torch.float8_e4m3fn), "scale": s["scale"], "back": s["back"]}
    if s["op"] == "norm":
        P.condensa_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, sum=s["sum"], y=s["y"], codes=s.get("Q"))
        return _only({"sum": s["sum"], "y": s["y"], "codes": s["q"], "scale": s["scale"]})
    if s["op"] == "norm-back":
        P.condensa_rms_norm_backward(s["dy"], s["h"], s["weight"], dsum=s["dsum"], eps=EPS, dx=s["dx"], dweight=s["dweight"], codes=s.get("Q"),
                                     workspace=s["workspace"])
        return _only({"dx": s["dx"], "dweight": s["dweight"], "codes": s["q"], "scale": s["scale"]})
    call = P.condensa_project_fp8 if s["op"] == "project" else P.condensa_project_fp8_backward
    call(s["X"], s["W"], s["y"], workspace=s["workspace"])
    return {"y": s["y"]}


def _only(out):
    """What is there; codes as the values they stand for."""
    return {k: v.view(torch.float8_e4m3fn) if k == "codes" else v for k, v in out.items() if v is not None}


def _in_blocks(x, block_rows):
    """[row blocks, block_rows, column blocks, 128], zeros past the ends."""
    R, C = x.shape
    x = torch.nn.functional.pad(x, (0, _blocks(C) * BLOCK - C, 0, -R % block_rows))
    return x.view(-1, block_rows, _blocks(C), BLOCK)


def _encode(x, block_rows):
    R, C = x.shape
    x = _in_blocks(x.float(), block_rows)
    size = x.abs()
    top = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax((1, 3), keepdim=True)
    kept = top >= 2.0 ** -100
    q = x.double() * 448 / torch.where(kept, top, torch.full_like(top, math.inf)).double()
    above = torch.nan_to_num(q / torch.frexp(q).mantissa, nan=0.0)       # 64 bits: many quotients lie next to the middle of two codes, or on it
    step = above.clamp(min=2.0 ** -5) / 16
    codes = ((q / step).round() * step).clamp(-448, 448).to(torch.float8_e4m3fn)
    scale = torch.where(kept, top / 448, torch.zeros_like(top))
    return codes.view(-1, _blocks(C) * BLOCK)[:R, :C], scale.view(-1, _blocks(C))


def _decode(q, scale, block_rows):
    R, C = q.shape
    by = scale.repeat_interleave(block_rows, 0)[:R].repeat_interleave(BLOCK, 1)[:, :C]
    return q.view(torch.float8_e4m3fn).float() * by


def _plain_codec(s):
    codes, scale = _encode(s["x"], s["block_rows"])
    return {"codes": codes, "scale": scale, "back": _decode(codes.view(torch.uint8), scale, s["block_rows"]).to(s["type"])}


def _with_codes(s, out, x):
    if s["q"] is not None:
        out["codes"], out["scale"] = _encode(x, 1)
    return out


def _plain_norm(s):
    out = {}
    h = s["x"]
    if s["residual"] is not None:
        h = out["sum"] = (h.float() + s["residual"].float()).to(s["type"])
    h = h.float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    if s["y"] is not None:
        out["y"] = y.to(s["type"])
    return _with_codes(s, out, y)


def _plain_norm_back(s):
    h, dy = s["h"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    u = h * r
    g = dy * s["weight"].float()
    dx = r * (g - u * (g * u).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return _with_codes(s, {"dx": dx.to(s["type"]), "dweight": (dy * u).sum(0)}, dx)


def _plain_project(s):
    return {"y": (_decode(s["x"], s["x_scale"], 1) @ _decode(s["w"], s["w_scale"], BLOCK).t()).to(s["type"])}


def _plain_back(s):
    return {"y": (_decode(s["x"], s["x_scale"], 1) @ _decode(s["w"], s["w_scale"], BLOCK)).to(s["type"])}


PLAIN = {"codec": _plain_codec, "norm": _plain_norm, "norm-back": _plain_norm_back, "project": _plain_project, "back": _plain_back}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    if case["op"] == "codec":
        n, scales = case["rows"] * case["cols"], 4 * -(-case["rows"] // case["block_rows"]) * _blocks(case["cols"])
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": n * (2 * size + 2) + 2 * scales, "flops": 3 * n}
    if case["op"] in ("norm", "norm-back"):
        T, n = case["tokens"], case["width"]
        codes = T * (n + 4 * _blocks(n)) if case["codes"] else 0
        weight = n * (4 if case["weight"] == "f32" else 2)
        if case["op"] == "norm":
            return {"bytes": 2 * T * n * (1 + 2 * case["residual"] + case["wide"]) + codes + weight, "flops": T * n * (4 + case["residual"] + 2 * case["codes"])}
        return {"bytes": 2 * T * n * (3 + case["residual"]) + codes + weight + 4 * n, "flops": T * n * (10 + case["residual"] + 2 * case["codes"])}
    T, K, N = case["tokens"], case["n_in"], case["n_out"]
    n_sum, n_wide = (K, N) if case["op"] == "project" else (N, K)
    return {"bytes": T * n_sum + 4 * T * _blocks(n_sum) + N * K + 4 * _blocks(N) * _blocks(K) + 2 * T * n_wide, "flops": 2 * T * N * K}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _exact_codes(x, block_rows):
    """Values of the e4m3 grid next to x / scale: multiples of 2^(e-3), e the exponent of x / scale and at least -6; the scales; their products."""
    R, C = x.shape
    pad = torch.zeros(_blocks(R) * BLOCK if block_rows > 1 else R, _blocks(C) * BLOCK, device=DEVICE, dtype=torch.float64)
    pad[:R, :C] = x
    tiles = pad.unfold(0, block_rows, block_rows).unfold(1, BLOCK, BLOCK)
    finite = torch.nan_to_num(tiles.abs(), nan=0.0, posinf=0.0)
    most = finite.amax((2, 3))
    most = torch.where(most < 2.0 ** -100, torch.zeros_like(most), most)
    each = most.repeat_interleave(block_rows, 0).repeat_interleave(BLOCK, 1)[:R, :C]
    q = torch.where(each > 0, 448 * x.abs() / torch.where(each > 0, each, torch.ones_like(each)), torch.zeros_like(x))
    borders = torch.tensor([2.0 ** e for e in range(-5, 9)], device=DEVICE, dtype=torch.float64)
    steps = torch.tensor([2.0 ** e for e in range(-9, 6)], device=DEVICE, dtype=torch.float64)
    step = steps[torch.bucketize(q, borders, right=True)]
    q = torch.copysign((torch.round(q / step) * step).clamp(max=448), x)
    return q, most / 448, q * each / 448


def _exact_norm(case, s):
    h = s["x"]
    out = {}
    if s["residual"] is not None:
        out["sum"] = h.double() + s["residual"].double()
        h = out["sum"].to(s["type"])
    h = h.double()
    y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["width"] + EPS) * s["weight"].double()[None]
    if case["wide"]:
        out["y"] = y
    if case["codes"]:
        out["codes"], out["scale"], _ = _exact_codes(y, 1)
    return out


def _exact_norm_back(case, s):
    h, dy, w, n = s["h"].double(), s["dy"].double(), s["weight"].double(), case["width"]
    ms = h.square().sum(1, keepdim=True) / n + EPS
    g = dy * w
    dx = g / ms.sqrt() - h * (g * h).sum(1, keepdim=True) / (n * ms * ms.sqrt())
    if s["dsum"] is not None:
        dx = dx + s["dsum"].double()
    out = {"dx": dx, "dweight": (dy * h / ms.sqrt()).sum(0)}
    if case["codes"]:
        out["codes"], out["scale"], _ = _exact_codes(dx, 1)
    return out


def _e4m3_value(byte):
    """The value of a code: 2^(e-7) (1 + m/8), or 2^-6 m/8 where e is 0."""
    e, m = byte >> 3 & 15, (byte & 7).double()
    power = torch.tensor([2.0 ** max(i - 7, -6) for i in range(16)], device=DEVICE, dtype=torch.float64)
    size = power[e] * ((e > 0).double() + m / 8)
    return torch.where(byte >= 128, -size, size)


def _exact_product(case, s):
    def values(q, scale, block_rows):
        v = _e4m3_value(q.int())
        at = torch.arange(v.shape[0], device=DEVICE)[:, None].div(block_rows, rounding_mode="floor"), torch.arange(v.shape[1], device=DEVICE)[None].div(BLOCK, rounding_mode="floor")
        return v * scale.double()[at]

    x, w = values(s["x"], s["x_scale"], 1), values(s["w"], s["w_scale"], BLOCK)
    return {"y": torch.mm(x, w.t().contiguous() if case["op"] == "project" else w)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "codec":
        codes, scale, back = _exact_codes(s["x"].double(), case["block_rows"])
        return {"codes": codes, "scale": scale, "back": back}
    if case["op"] == "norm":
        return _exact_norm(case, s)
    return _exact_norm_back(case, s) if case["op"] == "norm-back" else _exact_product(case, s)
