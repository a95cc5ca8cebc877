"""Cases of the operators on device tensors: what a program that keeps its rows and weights in 4 microscaled bits, and
rotates its queries and keys, calls of `paper_2510_23264_amd`.

A case names one operator and its sizes:

  quantize   mx4_quantize of a tensor the program holds (activation rows, or a weight master [k][n] by its columns), then
             mx4_dequantize of the codes: what the 4 bits stand for, in bfloat16, which holds them exactly
  product    mx4_gemm of quantised rows and quantised weights, with the bias and the residual a layer adds
  rotary     rotary of queries and keys that lie side by side in the rows of a projection's result

The plain forms compute the same from the formulas with elementary torch operations.  Values: normal activations whose
channels differ in size (a few are much larger than the rest, as in trained models), rows of padding that are zero, weights of
standard deviation 0.02.  Sizes are those of the model shapes this repository's workloads have, and odd ones.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MAX_FLOPS = 2.0 * 8192 * 11008 * 4096          # of the largest listed product
MAX_BYTES = 16384 * 4096 * (2 + 2 + 2 * 17 / 32)       # of the largest listed streaming case, about


def listed():
    return [
        # the activation row of one token on its way into a 4096-wide layer: launches are all of it
        dict(name="quantize_token_4096", op="quantize", rows=1, cols=4096, type="bf16", by="rows"),
        # normalised rows of the GPT-2-small shape's prompt batch, in the engine's own fp32
        dict(name="quantize_800x768", op="quantize", rows=800, cols=768, type="f32", by="rows"),
        # a long prefill's activations
        dict(name="quantize_16384x4096", op="quantize", rows=16384, cols=4096, type="bf16", by="rows"),
        # an MLP master [4096][11008] at set-up: blocks run down its columns
        dict(name="quantize_weights_11008x4096", op="quantize", rows=11008, cols=4096, type="f32", by="columns"),
        # one token through a square projection, bias and residual: the weights' bytes are all of it
        dict(name="product_token_4096x4096", op="product", m=1, n=4096, k=4096, type="bf16", bias=True, residual=True),
        # a ragged handful of tokens into the gate of a wide MLP
        dict(name="product_19x11008x4096", op="product", m=19, n=11008, k=4096, type="f16", bias=False, residual=False),
        # queries, keys and values of the GPT-2-small shape's prompt batch, fp32 as the engine keeps them
        dict(name="product_800x2304x768", op="product", m=800, n=2304, k=768, type="f32", bias=True, residual=False),
        # unembedding of the last positions of that batch: an odd number of columns
        dict(name="product_50x50257x768", op="product", m=50, n=50257, k=768, type="f32", bias=False, residual=False),
        # a long prefill through a wide MLP matrix: the matrix cores are all of it
        dict(name="product_8192x11008x4096", op="product", m=8192, n=11008, k=4096, type="bf16", bias=True, residual=True),
        # the next token of a few sequences, far into their contexts
        dict(name="rotary_4_tokens", op="rotary", tokens=4, heads=40, gap=8, d=128, rot=128, type="bf16", layout="half",
             inverse=False, scaling="bands", factor=8.0, theta=500000.0, far=120000),
        # a prefill's queries and keys between the values they share rows with
        dict(name="rotary_8192_tokens", op="rotary", tokens=8192, heads=40, gap=8, d=128, rot=128, type="bf16", layout="half",
             inverse=False, scaling="none", factor=1.0, theta=10000.0, far=8192),
        # a quarter of each head, neighbouring elements paired, the gradient's direction, fp32 and an odd number of tokens
        dict(name="rotary_3001_inverse", op="rotary", tokens=3001, heads=24, gap=12, d=64, rot=16, type="f32",
             layout="interleaved", inverse=True, scaling="linear", factor=4.0, theta=10000.0, far=32768),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "rotary"])
    kind = rng.choice(list(TYPES))
    if op == "quantize":
        by = rng.choice(["rows", "rows", "columns"])
        rows = _log(rng, 1, 32768)
        cols = _log(rng, 1, 16384)
        c = dict(op=op, rows=rows, cols=cols, type=kind, by=by)
        while work(c)["bytes"] > MAX_BYTES:
            c["rows"] = c["rows"] * 2 // 3
        return c
    if op == "product":
        c = dict(op=op, m=_log(rng, 1, 16384), n=_log(rng, 1, 50257), k=_log(rng, 1, 16384), type=kind,
                 bias=rng.random() < 0.5, residual=rng.random() < 0.5)
        while work(c)["flops"] > MAX_FLOPS or work(c)["bytes"] > MAX_BYTES:
            big = "m" if c["m"] > 64 else "n"
            c[big] = c[big] * 2 // 3
        return c
    d = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, 256])
    rot = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
    scaling = rng.choice(["none", "linear", "base", "bands"])
    if scaling == "base" and rot < 4:
        scaling = "linear"
    far = _log(rng, 16, 1 << 20)
    c = dict(op=op, tokens=_log(rng, 1, 32768), heads=rng.randint(1, 64), gap=rng.choice([0, 0, 1, 8]), d=d, rot=rot, type=kind,
             layout=rng.choice(["half", "interleaved"]), inverse=rng.random() < 0.4, scaling=scaling,
             factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 16.0), 2), theta=rng.choice([10000.0, 500000.0, 1e6]), far=far)
    while work(c)["bytes"] > MAX_BYTES:
        c["tokens"] = max(1, c["tokens"] * 2 // 3)
    return c


def work(case):
    c = case
    if c["op"] == "quantize":       # the tensor, its codes and scales out and in again, the values
        n = c["rows"] * c["cols"]
        return {"bytes": n * (BYTES[c["type"]] + 2 * 17 / 32 + 2), "flops": 0}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        out = m * n * BYTES[c["type"]] * (2 if c["residual"] else 1)
        return {"bytes": (m + n) * k * 17 / 32 + out + (4 * n if c["bias"] else 0), "flops": 2.0 * m * n * k}
    n = c["tokens"] * c["heads"] * c["d"]
    return {"bytes": 2 * n * BYTES[c["type"]] + 8 * c["tokens"], "flops": 0}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols):
    """Rows whose channels differ in size; a few channels are much larger; about one row in fifty is padding."""
    size = torch.exp(0.7 * _normal(g, cols))
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, size * 30, size)
    x = _normal(g, rows, cols) * size
    if rows > 8:
        x = x * (torch.rand(rows, 1, generator=g, device="cuda") > 0.02)
    return x


GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _blocks(x):
    """[r][c] in fp32 -> (signed values on the 4-bit grid [r][b][32], exponents of the scales [r][b])."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 32)).reshape(r, -1, 32)
    top = x.abs().amax(2)
    e = torch.where(top > 0, torch.clamp(torch.frexp(top)[1] - 3, min=-127), torch.zeros_like(top, dtype=torch.int32))
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(torch.clamp(torch.round(a / step) * step, max=6.0), y), e


def _held(x):
    """Rows as the library holds them: two codes a byte, one scale byte per 32, rows padded to 256 elements."""
    q, e = _blocks(x)
    pad = -q.shape[1] % 8
    code = torch.zeros(q.shape, dtype=torch.uint8, device=q.device)
    for i, v in enumerate(GRID):
        code += (q.abs() == v).to(torch.uint8) * i
    code += torch.signbit(q).to(torch.uint8) * 8
    code = torch.nn.functional.pad(code, (0, 0, 0, pad)).reshape(q.shape[0], -1, 2)
    scale = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, pad), value=127)
    return (code[..., 0] | code[..., 1] << 4).contiguous(), scale.contiguous()


def _frequencies(c):
    """Radians a position, in 64 bits."""
    r, s = c["rot"], c["factor"]
    theta = c["theta"] * s ** (r / (r - 2)) if c["scaling"] == "base" else c["theta"]
    f = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if c["scaling"] == "linear":
        f = [v / s for v in f]
    if c["scaling"] == "bands":
        g = [min(1.0, max(0.0, (8192 * v / (2 * math.pi) - 1.0) / 3.0)) for v in f]
        f = [v * (w + (1 - w) / s) for v, w in zip(f, g)]
    return f


def _inputs(c, seed):
    g = _generator(seed)
    if c["op"] == "quantize":
        if c["by"] == "rows":
            return (_activations(g, c["rows"], c["cols"]).to(TYPES[c["type"]]),)
        return ((0.02 * _normal(g, c["cols"], c["rows"])).to(TYPES[c["type"]]),)
    if c["op"] == "product":
        m, n, k, t = c["m"], c["n"], c["k"], TYPES[c["type"]]
        a, w = _held(_activations(g, m, k)), _held(0.02 * _normal(g, n, k))
        bias = 0.1 * _normal(g, n) if c["bias"] else None
        residual = (2 * _normal(g, m, n)).to(t) if c["residual"] else None
        return a, w, bias, residual
    rows = _normal(g, c["tokens"], c["heads"] + c["gap"], c["d"]).to(TYPES[c["type"]])
    # runs of neighbouring positions, as the sequences of a ragged batch have them
    start = torch.randint(0, c["far"], (c["tokens"] // 700 + 1,), generator=g, device="cuda")
    t = torch.arange(c["tokens"], device="cuda")
    return rows, start[t // 700] + t % 700


def prepare(case, seed):
    state = dict(case=case, inputs=_inputs(case, seed))
    if own:
        import paper_2510_23264_amd as P
        state["P"] = P
        if case["op"] == "product":
            (ac, asc), (wc, wsc), _, _ = state["inputs"]
            state["a"] = P.Mx4(ac, asc, case["k"])
            state["w"] = P.Mx4(wc, wsc, case["k"])
        if case["op"] == "rotary":
            state["table"] = P.rotary_table(case["rot"], theta=case["theta"], scaling=case["scaling"], factor=case["factor"],
                                            original=8192, turns=(1.0, 4.0), device="cuda")
    elif case["op"] == "rotary":
        state["table"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    c, P = state["case"], state["P"]
    if c["op"] == "quantize":
        q = P.mx4_quantize(state["inputs"][0], by=c["by"])
        return P.mx4_dequantize(q, dtype=torch.bfloat16)
    if c["op"] == "product":
        _, _, bias, residual = state["inputs"]
        return P.mx4_gemm(state["a"], state["w"], bias=bias, residual=residual, dtype=TYPES[c["type"]])
    rows, positions = state["inputs"]
    return P.rotary(rows[:, :c["heads"]], positions, state["table"], layout=c["layout"], inverse=c["inverse"])


def _values(held):
    """fp32 values of codes and scales, padding included."""
    codes, scales = held
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float32, device=codes.device)
    v = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), dim=-1).reshape(codes.shape[0], -1, 32)
    return torch.ldexp(v, (scales.to(torch.int32) - 127)[..., None]).reshape(codes.shape[0], -1)


def _run_plain(state):
    c = state["case"]
    if c["op"] == "quantize":
        x = state["inputs"][0].float()
        if c["by"] == "columns":
            x = x.t().contiguous()
        q, e = _blocks(x)
        return torch.ldexp(q, e[..., None]).reshape(x.shape[0], -1)[:, :x.shape[1]].to(torch.bfloat16)
    if c["op"] == "product":
        a, w, bias, residual = state["inputs"]
        y = torch.matmul(_values(a), _values(w).t())
        if bias is not None:
            y = y + bias
        if residual is not None:
            y = y + residual.float()
        return y.to(TYPES[c["type"]])
    rows, positions = state["inputs"]
    angle = positions.double()[:, None] * state["table"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["inverse"]:
        sin = -sin
    x, r = rows[:, :c["heads"]].float(), c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    return torch.cat((turned, x[..., r:]), dim=-1).to(rows.dtype)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    c = case
    if c["op"] == "quantize":
        x = _inputs(c, seed)[0].double()
        x = x if c["by"] == "rows" else x.t()
        out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        edges = torch.tensor([(a + b) / 2 for a, b in zip(GRID, GRID[1:])], dtype=torch.float64, device=x.device)
        grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
        for at in range(0, x.shape[1], 32):
            part = x[:, at:at + 32]
            top = part.abs().max(dim=1, keepdim=True).values
            # the largest power of two not above the block's largest value, a quarter of it (bit-exact through frexp)
            unit = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.clamp(torch.frexp(top)[1] - 3, min=-127)),
                               torch.ones_like(top))
            y = part.abs() / unit
            # on a border between two grid values the one with an even code: codes 1, 3, 5 give way to their neighbours
            low = torch.searchsorted(edges, y.contiguous())                   # borders strictly below y
            tie = (y == edges[low.clamp(max=6)]) & (low < 7) & (low % 2 == 1)
            out[:, at:at + 32] = torch.copysign(grid[low + tie.long()] * unit, part)
        return out
    if c["op"] == "product":
        (ac, asc), (wc, wsc), bias, residual = _inputs(c, seed)

        def wide(codes, scales):
            both = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.int64, device=codes.device)
            both[:, 0::2], both[:, 1::2] = codes & 15, codes >> 4
            m, e = both & 1, both >> 1 & 3                                  # one mantissa bit, two exponent bits, bias 1
            mag = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * 2.0 ** (e - 1).double())
            sign = 1 - 2 * (both >> 3 & 1).double()
            return sign * mag * (2.0 ** (scales.double() - 127)).repeat_interleave(32, dim=1)

        a, w = wide(ac, asc), wide(wc, wsc)
        y = torch.zeros(c["m"], c["n"], dtype=torch.float64, device=a.device) if bias is None else \
            bias.double().repeat(c["m"], 1)
        for at in range(0, a.shape[1], 2048):
            y += a[:, at:at + 2048] @ w[:, at:at + 2048].t().contiguous()
        return y if residual is None else y + residual.double()
    rows, positions = _inputs(c, seed)
    out = rows[:, :c["heads"]].double().clone()
    x = rows.double()
    for i, f in enumerate(_frequencies(c)):
        ia, ib = (i, i + c["rot"] // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        turn = torch.polar(torch.ones_like(positions, dtype=torch.float64), positions.double() * (-f if c["inverse"] else f))
        z = torch.complex(x[:, :c["heads"], ia].contiguous(), x[:, :c["heads"], ib].contiguous()) * turn[:, None]
        out[..., ia], out[..., ib] = z.real, z.imag
    return out
