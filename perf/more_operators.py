"""Performance cases of the operators around attention in a model that reads a pooled BEV map.

Five kinds of work, each calls of the package, channels last throughout:

  norm     ``rms_norm`` and ``rms_norm_add``: root-mean-square norm of every row, of x + residual
           with the sum handed on
  project  ``rms_norm_int8`` or ``rms_norm_add_int8``, then ``linear_int8``: a norm whose result is
           held in 8 bits with a scale for each row, read by the product that follows; serving
  linear   ``linear_int8``: a matrix product of 8-bit integers with a scale for each token and each
           output channel; serving
  rotary   ``rotary``: pairs of channels turned by angles that go with a token's position (along
           one axis, or the two or three of a map), interleaved or in halves, part of the head
  gate     ``gated_act``: act(gate) * value, the halves of a row, with what the backward needs kept
           as it is or in 8 bits (blocks of 32 channels that share a power of two)

``train`` asks for the outputs and the gradients of all inputs. ``run`` computes the operators from
elementary torch operations in 32 bits (angles in 64), or, where ``own`` is true, through the
package. ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_POSITIONS = {"i32": torch.int32, "i64": torch.int64, "f32": torch.float32}
_EPS = 1e-6
_BLOCK = 32     # channels that share an exponent


def _norm(**over):
    return {"op": "norm", "train": True, "rows": 600, "channels": 256, "dtype": "bf16", "out": "bf16",
            "residual": True, **over}


def _project(**over):
    return {"op": "project", "train": False, "rows": 129600, "channels": 80, "features": 256, "dtype": "bf16",
            "out": "bf16", "residual": True, **over}


def _linear(**over):
    return {"op": "linear", "train": False, "rows": 16896, "channels": 2048, "features": 4096, "out": "bf16",
            "bias": False, **over}


def _rotary(**over):
    return {"op": "rotary", "train": False, "batch": 1, "tokens": 129600, "heads": 4, "dim": 32, "pairs": 16,
            "axes": 1, "interleaved": False, "positions": "i32", "dtype": "bf16", "packed": False,
            "amplitude": 1.0, **over}


def _gate(**over):
    return {"op": "gate", "train": True, "rows": 129600, "features": 320, "act": "silu", "dtype": "bf16",
            "checkpoint": True, **over}


def listed():
    return [
        # a training step of the queries' norm before attention, two samples of 300 object queries
        _norm(name="norm_queries", dtype="f16", out="f16"),
        # a training step of the norm of every cell of four maps, the residual stream handed on
        _norm(name="norm_map", rows=4 * 360 * 360, channels=80),
        # one token of a language model asks: norm and projection, where latency counts
        _project(name="project_token", rows=1, channels=1024, features=4096),
        # the cells of the typical frame's map become keys and values: online inference
        _project(name="project_map"),
        # sixty-four requests' tokens through a feed-forward layer: the weights are what is read
        _linear(name="linear_batch", rows=64, channels=4096, features=2048, out="f16", bias=True),
        # sizes that divide nothing, the result in fp32
        _linear(name="linear_odd", rows=1111, channels=331, features=517, out="f32", bias=True),
        # the pixels of six cameras of 32x88 features through a wide layer
        _linear(name="linear_pixels"),
        # one token each of eight requests, far into their contexts, queries and keys in one projection
        _rotary(name="rotary_token", batch=8, tokens=1, heads=10, dim=64, pairs=32, positions="i64"),
        # a training step on the map's cells as keys, at metric positions along two axes, a view of packed keys and values
        _rotary(name="rotary_cells", train=True, axes=2, positions="f32", packed=True),
        # a captioner's prompts, half of each head turned, interleaved, scaled for a longer context
        _rotary(name="rotary_prompt", batch=8, tokens=1024, heads=16, dim=128, pairs=32, interleaved=True,
                dtype="f16", amplitude=1.14),
        # a training step of the object queries' feed-forward layer in fp32, nothing rounded
        _gate(name="gate_queries", rows=600, features=1024, act="gelu", dtype="f32", checkpoint=False),
        # a training step of a feed-forward layer over the cells of a map, what it keeps in 8 bits
        _gate(name="gate_map"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "project", "linear", "rotary", "gate"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    while True:
        if op == "norm":
            case = _norm(train=rng.random() < 0.6, rows=_log(rng, 1, 4 * 360 * 360),
                         channels=rng.choice([80, 128, 256, 1024, _log(rng, 4, 4096)]), dtype=dtype,
                         out=rng.choice([dtype, "f32", "bf16"]), residual=rng.random() < 0.6)
            if case["rows"] * case["channels"] <= 4 * 360 * 360 * 80:
                return case
        elif op in ("project", "linear"):
            sizes = {"rows": rng.choice([1, _log(rng, 1, 129600)]),
                     "channels": rng.choice([80, 256, 1024, 2048, _log(rng, 16, 4096)]),
                     "features": rng.choice([80, 256, 1024, 2048, _log(rng, 16, 4096)])}
            if op == "project":
                case = _project(dtype=dtype, out=rng.choice(["bf16", "f16"]), residual=rng.random() < 0.6, **sizes)
            else:
                case = _linear(out=dtype, bias=rng.random() < 0.5, **sizes)
            if work(case)["flops"] <= 2.8e11 and case["rows"] * max(case["channels"], case["features"]) <= 7e7:
                return case
        elif op == "rotary":
            axes = rng.choice([1, 1, 2, 3])
            pairs = axes * rng.choice([4, 8, 16, rng.randint(1, 24)])
            case = _rotary(train=rng.random() < 0.5, batch=_log(rng, 1, 8), tokens=rng.choice([1, _log(rng, 1, 129600)]),
                           heads=rng.choice([1, 2, 4, 8, rng.randint(1, 16)]),
                           dim=rng.choice([2 * pairs, 2 * pairs, 64, 128, 2 * pairs + rng.randint(1, 16)]), pairs=pairs,
                           axes=axes, interleaved=rng.random() < 0.5, positions=rng.choice(["i32", "i64", "f32"]),
                           dtype=dtype, packed=rng.random() < 0.5, amplitude=rng.choice([1.0, rng.uniform(1, 1.5)]))
            if 2 * pairs <= case["dim"] <= 128 and \
                    case["batch"] * case["tokens"] * case["heads"] * case["dim"] <= 8 * 1024 * 16 * 128:
                return case
        else:
            case = _gate(train=rng.random() < 0.7, rows=_log(rng, 1, 129600),
                         features=rng.choice([320, 512, 1024, _log(rng, 1, 4096)]),
                         act=rng.choice(["none", "relu", "silu", "gelu"]), dtype=dtype, checkpoint=rng.random() < 0.6)
            if case["rows"] * case["features"] <= 129600 * 320:
                return case


def work(case):
    size, out = _BYTES.get(case.get("dtype")), _BYTES.get(case.get("out"))
    if case["op"] == "norm":
        n, c = case["rows"] * case["channels"], case["channels"]
        # x, y; the residual and the sum; for a step dy, dx, and the gradient of the sum
        step = n * (size + out) * (2 if case["train"] else 1) + 4 * c * (2 if case["train"] else 1)
        return {"bytes": step + n * size * case["residual"] * (3 if case["train"] else 2),
                "flops": n * (16 if case["train"] else 5)}
    if case["op"] in ("project", "linear"):
        m, k, n = case["rows"], case["channels"], case["features"]
        read = m * k * (size * (1 + 2 * case["residual"]) if case["op"] == "project" else 1)
        return {"bytes": read + n * k + m * n * out + 4 * (m + n), "flops": 2 * m * n * k}
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"]
        n = rows * case["heads"] * case["dim"]
        place = _POSITIONS[case["positions"]].itemsize * case["axes"] * rows
        # x, out, positions; for a step their gradients
        return {"bytes": (2 * n * size + place) * (2 if case["train"] else 1),
                "flops": (3 * n + 20 * rows * case["pairs"]) * (2 if case["train"] else 1)}
    n = case["rows"] * case["features"]
    # two halves, y; for a step dy and the gradients of both halves (what is kept in between is not counted)
    return {"bytes": n * size * (6 if case["train"] else 3), "flops": n * (20 if case["train"] else 8)}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype = _TORCH[case.get("dtype", "f32")]

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(shape, generator=gen, device=dev) * scale).to(to)

    def leaf(t):
        return t.detach().requires_grad_(case["train"])

    def held(rows, columns, scale):
        """Rows of 8-bit integers and their scales."""
        t = normal(rows, columns, scale=scale, to=torch.float32)
        step = t.abs().amax(1) / 127
        return torch.round(t / step[:, None]).to(torch.int8), step

    state = {"case": case}
    if case["op"] in ("norm", "project"):
        m, c = case["rows"], case["channels"]
        # rows of different size, as a residual stream has them
        loud = torch.exp(0.5 * torch.randn((m, 1), generator=gen, device=dev))
        state["x"] = leaf(normal(m, c))
        state["residual"] = leaf((normal(m, c, to=torch.float32) * loud).to(dtype)) if case["residual"] else None
        state["weight"] = leaf(1 + normal(c, scale=0.2, to=torch.float32))
        if case["train"]:
            state["dy"] = normal(m, c, to=_TORCH[case["out"]])
            state["dsum"] = normal(m, c) if case["residual"] else None
    if case["op"] in ("project", "linear"):
        k, n = case["channels"], case["features"]
        if case["op"] == "linear":
            state["x"], state["scale"] = held(case["rows"], k, 1.0)
        state["w"], state["w_scale"] = held(n, k, k ** -0.5)
        state["bias"] = normal(n, scale=0.2, to=torch.float32) if case.get("bias") else None
    if case["op"] == "rotary":
        b, n, h, d = (case[k] for k in ("batch", "tokens", "heads", "dim"))
        wide = normal(b, n, 2 if case["packed"] else 1, h, d, scale=2.0)
        state["x"] = leaf(wide[:, :, 0])
        shape = (b, n) if case["axes"] == 1 else (b, n, case["axes"])
        if case["positions"] == "f32":      # metres from the rig
            place = (torch.rand(shape, generator=gen, device=dev) - 0.5) * 108
        else:                               # a run of tokens that starts anywhere in a long context
            start = torch.randint(0, 1 << 20, (b,) + (1,) * (len(shape) - 1), generator=gen, device=dev)
            place = torch.arange(n, device=dev).view((1, n) + (1,) * (len(shape) - 2)) + start.expand(
                (b, 1) + shape[2:])
        state["positions"] = place.to(_POSITIONS[case["positions"]]).contiguous()
        per = case["pairs"] // case["axes"]
        state["frequencies"] = (10000.0 ** (-torch.arange(per, dtype=torch.float64, device=dev) / per)).repeat(
            case["axes"])
        if case["train"]:
            state["dy"] = normal(b, n, h, d)
    if case["op"] == "gate":
        # a few channels far above the others, as feed-forward layers have them
        loud = torch.exp(0.7 * torch.randn(2 * case["features"], generator=gen, device=dev))
        state["x"] = leaf((normal(case["rows"], 2 * case["features"], to=torch.float32) * loud).to(dtype))
        if case["train"]:
            state["dy"] = normal(case["rows"], case["features"])
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2205_13542_amd as bev
    c = s["case"]
    out = _TORCH.get(c.get("out"))
    if c["op"] == "norm":
        if not c["residual"]:
            y = bev.rms_norm(s["x"], s["weight"], eps=_EPS, out_dtype=out)
            return (y, *torch.autograd.grad(y, (s["x"], s["weight"]), s["dy"])) if c["train"] else y
        y, total = bev.rms_norm_add(s["x"], s["residual"], s["weight"], eps=_EPS, out_dtype=out)
        if not c["train"]:
            return y, total
        return (y, total, *torch.autograd.grad((y, total), (s["x"], s["weight"], s["residual"]), (s["dy"], s["dsum"])))
    if c["op"] == "project":
        if not c["residual"]:
            held, scale = bev.rms_norm_int8(s["x"], s["weight"], eps=_EPS)
            return bev.linear_int8(held, scale, s["w"], s["w_scale"], out_dtype=out)
        held, scale, total = bev.rms_norm_add_int8(s["x"], s["residual"], s["weight"], eps=_EPS)
        return bev.linear_int8(held, scale, s["w"], s["w_scale"], out_dtype=out), total
    if c["op"] == "linear":
        return bev.linear_int8(s["x"], s["scale"], s["w"], s["w_scale"], bias=s["bias"], out_dtype=out)
    if c["op"] == "rotary":
        y = bev.rotary(s["x"], s["positions"], s["frequencies"], interleaved=c["interleaved"],
                       amplitude=c["amplitude"])
        return (y, *torch.autograd.grad(y, (s["x"],), s["dy"])) if c["train"] else y
    y = bev.gated_act(s["x"], act=c["act"], checkpoint="int8" if c["checkpoint"] else None)
    return (y, *torch.autograd.grad(y, (s["x"],), s["dy"])) if c["train"] else y


@torch.no_grad()
def _run_plain(s):
    c = s["case"]
    return {"norm": _plain_norm, "project": _plain_project, "linear": _plain_linear, "rotary": _plain_rotary,
            "gate": _plain_gate}[c["op"]](s, c)


def _plain_sum(s):
    """The rows, and one over the root of their mean square."""
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    return h, ((h * h).mean(1, keepdim=True) + _EPS).rsqrt()


def _plain_norm(s, c):
    h, r = _plain_sum(s)
    unit = h * r
    y = (unit * s["weight"]).to(_TORCH[c["out"]])
    dtype = s["x"].dtype
    if not c["train"]:
        return (y, h.to(dtype)) if c["residual"] else y
    dy = s["dy"].float()
    dw = (dy * unit).sum(0)
    e = dy * s["weight"]
    dh = r * (e - unit * (e * unit).mean(1, keepdim=True))
    if not c["residual"]:
        return y, dh.to(dtype), dw
    dh = (dh + s["dsum"].float()).to(dtype)
    return y, h.to(dtype), dh, dw, dh


def _plain_project(s, c):
    h, r = _plain_sum(s)
    z = h * s["weight"]
    top = z.abs().amax(1, keepdim=True)
    held = torch.round(z * (127 / top))
    y = (held @ s["w"].float().t()) * (top * r / 127) * s["w_scale"]
    y = y.to(_TORCH[c["out"]])
    return (y, h.to(s["x"].dtype)) if c["residual"] else y


def _plain_linear(s, c):
    y = (s["x"].float() @ s["w"].float().t()) * s["scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_TORCH[c["out"]])


def _plain_turn(x, c, cos, sin):
    """x turned by angles of which cos and sin [b][n][1][pairs] are given."""
    x, p = x.float(), c["pairs"]
    turned, rest = x[..., :2 * p], x[..., 2 * p:]
    if c["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = turned[..., :p], turned[..., p:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, rest), -1)


def _plain_rotary(s, c):
    place = s["positions"].double()
    place = place.view(place.shape[0], place.shape[1], c["axes"]).repeat_interleave(c["pairs"] // c["axes"], 2)
    angle = (place * s["frequencies"])[:, :, None]
    cos, sin = (c["amplitude"] * angle.cos()).float(), (c["amplitude"] * angle.sin()).float()
    y = _plain_turn(s["x"], c, cos, sin).to(s["x"].dtype)
    if not c["train"]:
        return y
    return y, _plain_turn(s["dy"], c, cos, -sin).to(s["x"].dtype)


def _plain_held(x, f):
    """x as 8-bit integers times powers of two: blocks of 32 channels of each half share the least power
    of two whose 127-fold reaches their largest magnitude."""
    pad = -f % _BLOCK
    t = torch.nn.functional.pad(x.view(-1, 2, f), (0, pad)).view(x.shape[0], 2, -1, _BLOCK)
    part, power = torch.frexp(t.abs().amax(-1, keepdim=True))
    power = (power - 7 + (part > 127 / 128)).clamp(-126, 126)

    def two_to(e):      # from its bits: a computed power may be off in the last one
        return (e + 127 << 23).view(torch.float32)

    held = torch.round(t * two_to(-power)) * two_to(power)
    return held.view(x.shape[0], 2, -1)[..., :f].reshape(x.shape)


def _plain_act(g, act):
    """act(g) and its slope."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    return g, torch.ones_like(g)


def _plain_gate(s, c):
    x, f = s["x"].float(), c["features"]
    y = (_plain_act(x[:, :f], c["act"])[0] * x[:, f:]).to(s["x"].dtype)
    if not c["train"]:
        return y
    if c["checkpoint"]:
        x = _plain_held(x, f)
    a, slope = _plain_act(x[:, :f], c["act"])
    dy = s["dy"].float()
    return y, torch.cat((dy * x[:, f:] * slope, dy * a), 1).to(s["x"].dtype)


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "project": _exact_project, "linear": _exact_linear, "rotary": _exact_rotary,
            "gate": _exact_gate}[case["op"]](s, case)


def _exact_norm(s, c):
    """Through the definition's own differentiation."""
    leaves = [t.detach().double().requires_grad_() for t in (s["x"], s["weight"], s["residual"]) if t is not None]
    with torch.enable_grad():
        h = leaves[0] + leaves[2] if c["residual"] else leaves[0]
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / c["channels"] + _EPS) * leaves[1]
        outputs = (y, h) if c["residual"] else (y,)
        if c["train"]:
            grads = torch.autograd.grad(outputs, leaves, [s[d].double() for d in ("dy", "dsum")[:len(outputs)]])
    outputs = tuple(t.detach() for t in outputs)
    if c["train"]:
        return outputs + grads
    return outputs if c["residual"] else outputs[0]


def _exact_project(s, c):
    h = s["x"].double() + (s["residual"].double() if c["residual"] else 0)
    z = h / torch.sqrt(h.square().sum(1, keepdim=True) / c["channels"] + _EPS) * s["weight"].double()
    step = z.abs().amax(1, keepdim=True) / 127
    y = (torch.round(z / step) * step) @ (s["w"].double() * s["w_scale"].double()[:, None]).t().contiguous()
    return (y, h) if c["residual"] else y


def _exact_linear(s, c):
    y = (s["x"].double() * s["scale"].double()[:, None]) @ \
        (s["w"].double() * s["w_scale"].double()[:, None]).t().contiguous()
    return y + s["bias"].double() if c["bias"] else y


def _exact_rotary(s, c):
    """Pairs as complex numbers, turned by a product."""
    p = c["pairs"]
    place = s["positions"].double()
    if c["axes"] == 1:
        place = place[..., None]
    angle = torch.cat([place[..., a:a + 1] * f for a, f in enumerate(s["frequencies"].chunk(c["axes"]))], -1)
    turn = torch.polar(torch.full_like(angle, c["amplitude"]), angle)[:, :, None]

    def turned(x, by):
        x = x.double()
        pairs = x[..., :2 * p].unflatten(-1, (p, 2) if c["interleaved"] else (2, p))
        if not c["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
        if not c["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        return torch.cat((pairs.flatten(-2), x[..., 2 * p:]), -1)

    y = turned(s["x"], turn)
    return (y, turned(s["dy"], turn.conj())) if c["train"] else y


def _exact_gate(s, c):
    f = c["features"]
    x = s["x"].double()

    def forward(t):
        g, v = t[:, :f], t[:, f:]
        if c["act"] == "relu":
            g = torch.where(g > 0, g, 0)
        elif c["act"] == "silu":
            g = g * torch.sigmoid(g)
        elif c["act"] == "gelu":
            g = g * 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * v

    y = forward(x)
    if not c["train"]:
        return y
    if c["checkpoint"]:
        blocks = [x[:, half + first:half + min(first + _BLOCK, f)] for half in (0, f) for first in range(0, f, _BLOCK)]
        x = torch.cat([_exact_held(t) for t in blocks], 1)
    x = x.detach().requires_grad_()
    with torch.enable_grad():
        dx, = torch.autograd.grad(forward(x), x, s["dy"].double())
    return y, dx


def _exact_held(t):
    top = t.abs().amax(1, keepdim=True)
    # the exponent field of top / 127, and one more unless that is a power of two
    bits = (top / 127).view(torch.int64)
    unit = (((bits >> 52) + (bits & (1 << 52) - 1 != 0)) << 52).view(torch.float64)
    return torch.where(top > 0, torch.round(t / unit) * unit, 0.0)
