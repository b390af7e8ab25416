"""The AdamW step against binary32 arithmetic with one rounding per operation (bit for bit) and against binary64."""
import numpy as np
import pytest
import torch

import paper_1911_02497_amd as P
from adamw_reference import BLOCK, decode, encode, noise, step32, step64
from gpu_util import DEV, assert_bits_equal

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HYPER = dict(betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)


class Problem:
    """A list of tensors on the device with what the reference needs of it on the host."""

    def __init__(self, sizes, bits, grad="f32", penalty=(), codes=(), code_type="bf16", offset=0, seed=0):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits = sizes, bits

        def put(a, dtype=None):
            t = torch.from_numpy(np.ascontiguousarray(a))
            whole = torch.zeros(t.numel() + offset, dtype=dtype or t.dtype, device=DEV)
            whole[offset:] = t.to(DEV).to(whole.dtype)
            return whole[offset:]

        normal = lambda n, s: (rng.standard_normal(n) * s).astype(np.float32)  # noqa: E731
        self.w = [put(normal(n, 0.02)) for n in sizes]
        self.g = [put(normal(n, 1e-3), TYPES[grad]) for n in sizes]
        m0, r0 = [normal(n, 3e-4) for n in sizes], [np.abs(normal(n, 1e-3)) for n in sizes]
        self.ms = self.rs = None
        if bits == 32:
            self.m, self.v = [put(m) for m in m0], [put(r * r) for r in r0]
        else:
            em, er = [encode(m, None, False) for m in m0], [encode(r, None, True) for r in r0]
            self.m, self.v = [put(c) for c, _ in em], [put(c) for c, _ in er]
            self.ms, self.rs = ([torch.from_numpy(s).to(DEV) for _, s in e] for e in (em, er))
        self.theta = [put(normal(n, 0.02)) if i in penalty else None for i, n in enumerate(sizes)] if penalty else None
        self.lam = [put(normal(n, 1e-4)) if i in penalty else None for i, n in enumerate(sizes)] if penalty else None
        self.codes = [put(np.zeros(n, np.float32), TYPES[code_type]) if i in codes else None for i, n in enumerate(sizes)] if codes else None

    def table(self, **kw):
        if self.bits == 8:
            kw.update(exp_avg_scale=self.ms, exp_avg_sq_scale=self.rs)
        return P.adamw_table(self.w, self.g, self.m, self.v, theta=self.theta, lambdas=self.lam, codes=self.codes, **kw)

    def host(self):
        """Copies of everything, as lists of arrays (None where there is nothing)."""
        get = lambda ts: [None if t is None else t.float().cpu().numpy() if t.dtype != torch.uint8 else t.cpu().numpy()  # noqa: E731
                          for t in (ts or [None] * len(self.sizes))]
        return {k: get(getattr(self, k)) for k in ("w", "g", "m", "v", "ms", "rs", "theta", "lam", "codes")}

    def check(self, before, what, lr, step, mu=0.0, seed=None, grad_scale=None):
        after, blocks = self.host(), 0
        for i, n in enumerate(self.sizes):
            b = {k: v[i] for k, v in before.items()}
            m, v = b["m"], b["v"]
            if self.bits == 8:
                m, v = decode(m, b["ms"]), decode(v, b["rs"]) ** 2
            with np.errstate(all="ignore"):
                w, m, v, r = step32(b["w"], b["g"], m, v, lr, step, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"],
                                    b["theta"], b["lam"], mu, grad_scale)
            assert_bits_equal(after["w"][i], w, f"{what} w {i}")
            if self.bits == 32:
                assert_bits_equal(after["m"][i], m, f"{what} m {i}")
                assert_bits_equal(after["v"][i], v, f"{what} v {i}")
            else:
                bits = None if seed is None else noise(seed, blocks, n)
                for name, x, low in (("m", m, True), ("v", r, False)):
                    part = None if bits is None else (bits & np.uint64(0xFFFF) if low else bits >> np.uint64(16))
                    code, scale = encode(x, part, not low)
                    assert_bits_equal(after["ms" if low else "rs"][i], scale, f"{what} scale of {name} {i}")
                    bad = np.flatnonzero(after[name][i] != code)
                    assert bad.size == 0, f"{what} codes of {name} {i}: {bad.size} of {n}, first {bad[:4]}: {after[name][i][bad[:4]]}, not {code[bad[:4]]}"
            if b["codes"] is not None:
                want = torch.from_numpy(w).to(self.codes[i].dtype).float().numpy()
                assert np.array_equal(after["codes"][i], want), f"{what} copy {i}"
            blocks += -(-n // BLOCK)


SIZES = [[1], [255, 257], [256], [0, 5, 8191, 0, 8193, 100003], [2, 0], list(range(250, 330))]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[-1]}")
@pytest.mark.parametrize("bits,seed", [(32, None), (8, None), (8, 0x123456789ABCDEF0)])
def test_sizes(sizes, bits, seed):
    p = Problem(sizes, bits, penalty={0, 2}, codes={0, 1, 3})
    t = p.table()
    for step in (1, 2, 1000):
        before = p.host()
        P.condensa_lc_adamw_step(t, 1e-3, step, mu=1e-3, seed=None if seed is None else seed + step, **HYPER)
        p.check(before, f"step {step}", 1e-3, step, mu=1e-3, seed=None if seed is None else seed + step)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("code_type", ["f16", "bf16"])
def test_types_and_alignment(bits, grad, offset, code_type):
    p = Problem([700, 4096, 33], bits, grad=grad, penalty={1}, codes={0, 1}, code_type=code_type, offset=offset)
    before, t = p.host(), p.table()
    scale = torch.tensor([0.25], device=DEV)
    P.condensa_lc_adamw_step(t, 2e-3, 7, mu=0.5, grad_scale=scale, **HYPER)
    p.check(before, "step", 2e-3, 7, mu=0.5, grad_scale=0.25)


@pytest.mark.parametrize("bits,seed", [(32, None), (8, None), (8, 5)])
def test_special_gradients(bits, seed):
    """Zero gradients on zero states, infinities and NaN: a bad gradient spoils its own element and no other."""
    n = 1000
    p = Problem([n, n], bits)
    with torch.no_grad():
        p.g[0].zero_()
        p.m[0].zero_()
        p.v[0].zero_()
        p.g[1][3], p.g[1][300], p.g[1][301], p.g[1][302] = float("inf"), float("-inf"), float("nan"), 3e38
        p.g[1][900] = 1e-40
    before = p.host()
    P.condensa_lc_adamw_step(p.table(), 1e-3, 3, seed=seed, **HYPER)
    after = p.host()
    assert np.all(np.isfinite(after["w"][0]))
    good = np.ones(n, bool)
    good[[3, 300, 301]] = False
    assert np.all(np.isfinite(after["w"][1][good])) and not np.any(np.isfinite(after["w"][1][~good]))
    if bits == 8:
        assert np.all(np.isfinite(after["ms"][1])) and np.array_equal(np.flatnonzero((after["m"][1] & 0x7F) == 0x7F), [301])
        assert (after["m"][1][3] & 0x7F) == 0x7E and (after["m"][1][300]) == 0xFE
    else:
        b = {k: v[1] for k, v in before.items()}
        with np.errstate(all="ignore"):
            w, m, v, _ = step32(b["w"], b["g"], b["m"], b["v"], 1e-3, 3, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
        for name, x in (("w", w), ("m", m), ("v", v)):
            assert_bits_equal(after[name][1][good], x[good], name)


def test_against_binary64():
    """m, v and w as of the textbook formula.  Roundings on the way, each at most 2^-24 of the value it makes: m: two products, their
    constants and one sum, 5 of |b1 m| + |c1 g|; v: three products, constants and one sum, 6 of v; the quotient u: m's 5, half of
    v's 6, the root, its product and constant, the sum with eps and the division, 13; w: 13 + 2 for the constant and product of u,
    2 for those of the decay and one of the difference, each of what it rounds.  g = grad, so nothing is cancelled before."""
    p = Problem([50000], 32)
    b = p.host()
    P.condensa_lc_adamw_step(p.table(), 1e-3, 10, **HYPER)
    a, h = p.host(), 2.0 ** -24
    w, m, v = step64(b["w"][0], b["g"][0], b["m"][0], b["v"][0], 1e-3, 10, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
    size_m = 0.9 * np.abs(b["m"][0].astype(np.float64)) + 0.1 * np.abs(b["g"][0].astype(np.float64))
    assert np.all(np.abs(a["m"][0] - m) <= 5 * h * size_m)
    assert np.all(np.abs(a["v"][0] - v) <= 6 * h * v)
    move = 1e-3 * size_m / (1 - 0.9 ** 10) / (np.sqrt(v / (1 - 0.999 ** 10)) + 1e-8)
    assert np.all(np.abs(a["w"][0] - w) <= 1.01 * h * (15 * move + 2 * np.abs(b["w"][0]) + np.abs(w)))


@pytest.mark.parametrize("stochastic", [True, False])
def test_stochastic_rounding_keeps_the_mean(stochastic):
    """A step moves the root of the second moment by a fraction of the distance of two codes.  With constant gradients of 1e-3, v goes
    from r0^2 towards 1e-6 as r0^2 0.99^k + 1e-6 (1 - 0.99^k); stochastic codes follow (their variance, of codes 6 to 12 % apart, adds
    about 1 % to v), codes to nearest stay.  Element 0 of every block has gradients and a root of 3e-3, which fixes the scale."""
    n, steps = 1 << 16, 400
    first = np.arange(n) % BLOCK == 0
    c, s = encode(np.where(first, 3e-3, 2e-3).astype(np.float32), None, True)
    r0 = decode(c, s)[1]
    w, g = torch.zeros(n, device=DEV), torch.from_numpy(np.where(first, 3e-3, 1e-3).astype(np.float32)).to(DEV)
    m, v = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.from_numpy(c).to(DEV)
    ms, vs = torch.zeros(n // BLOCK, device=DEV), torch.from_numpy(s).to(DEV)
    t = P.adamw_table([w], [g], [m], [v], exp_avg_scale=[ms], exp_avg_sq_scale=[vs])
    for k in range(steps):
        P.condensa_lc_adamw_step(t, 0.0, 1 + k, betas=(0.9, 0.99), seed=1000 + k if stochastic else None)
    mean = decode(v.cpu().numpy(), vs.cpu().numpy()).astype(np.float64)[~first].mean()
    want = np.sqrt(r0 ** 2 * 0.99 ** steps + 1e-6 * (1 - 0.99 ** steps))
    if stochastic:
        assert abs(mean / want - 1) < 0.03, (mean, want)
    else:
        assert abs(mean / r0 - 1) < 1e-3, (mean, r0)


@pytest.mark.parametrize("bits", [32, 8])
def test_streams_and_graphs(bits):
    """A captured step replays with eager steps of other tensors between, on a stream of its own."""
    p, q = Problem([5000, 300], bits, codes={0}), Problem([777], bits)
    tp, tq = p.table(), q.table()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    before = p.host()
    with torch.cuda.graph(g, stream=s):
        P.condensa_lc_adamw_step(tp, 1e-3, 5, seed=9 if bits == 8 else None, stream=torch.cuda.current_stream(), **HYPER)
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        p.check(before, f"replay {k}", 1e-3, 5, seed=9 if bits == 8 else None)
        before = p.host()
        other = q.host()
        P.condensa_lc_adamw_step(tq, 1e-3, 1 + k, **HYPER)
        torch.cuda.synchronize()
        q.check(other, f"eager {k}", 1e-3, 1 + k)


def test_beyond_32_bits():
    """One tensor of 2^32 + 999 elements with states in 8 bits: its last blocks are right, the first of the next tensor too."""
    n, tail = (1 << 32) + 999, 5000
    sizes = [n, 300]
    w, g = [torch.zeros(k, device=DEV) for k in sizes], [torch.zeros(k, device=DEV, dtype=torch.bfloat16) for k in sizes]
    m, v = ([torch.zeros(k, dtype=torch.uint8, device=DEV) for k in sizes] for _ in range(2))
    ms, vs = ([torch.zeros(-(-k // BLOCK), device=DEV) for k in sizes] for _ in range(2))
    torch.manual_seed(3)
    for t in range(2):
        k = min(tail, sizes[t])
        w[t][-k:] = torch.randn(k, device=DEV) * 0.02
        g[t][-k:] = (torch.randn(k, device=DEV) * 1e-3).bfloat16()
    before = [(w[t][-tail:].cpu().numpy(), g[t][-tail:].float().cpu().numpy()) for t in range(2)]
    table = P.adamw_table(w, g, m, v, exp_avg_scale=ms, exp_avg_sq_scale=vs)
    P.condensa_lc_adamw_step(table, 1e-3, 1, seed=77 << 32 | 5, **HYPER)
    for t in range(2):
        wb, gb = before[t]
        k = len(wb)
        wn, mn, vn, r = step32(wb, gb, np.zeros(k, np.float32), np.zeros(k, np.float32), 1e-3, 1, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
        assert_bits_equal(w[t][-k:].cpu(), wn, "w")
        start = (sizes[t] - k) // BLOCK * BLOCK + (BLOCK if t == 0 else 0)      # the first whole block of the part looked at
        cut = start - (sizes[t] - k)
        bits = noise(77 << 32 | 5, (-(-n // BLOCK) if t else 0) + start // BLOCK, k - cut)
        code, scale = encode(mn[cut:], bits & np.uint64(0xFFFF), False)
        assert np.array_equal(m[t][start:].cpu().numpy(), code)
        assert_bits_equal(ms[t][start // BLOCK:].cpu(), scale, "scale")
        code, scale = encode(r[cut:], bits >> np.uint64(16), True)
        assert np.array_equal(v[t][start:].cpu().numpy(), code)
    assert not bool(w[0][: 1 << 20].any()) and not bool(m[0][1 << 31:(1 << 31) + (1 << 20)].any())


def test_a_seed_decides_nothing_about_states_in_32_bits():
    p, q = Problem([700, 33], 32), Problem([700, 33], 32)
    P.condensa_lc_adamw_step(p.table(), 1e-3, 2, seed=1 << 40, **HYPER)
    P.condensa_lc_adamw_step(q.table(), 1e-3, 2, **HYPER)
    for a, b in zip(p.w + p.m + p.v, q.w + q.m + q.v):
        assert torch.equal(a, b)
