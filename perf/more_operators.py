"""Operators of residual blocks of an answer head, and of the step that trains them, as measurable cases.

A head of depth is made of residual blocks: the rows are normalised, widened by a gated pair of projections, narrowed by a linear layer
and added to what came in.  Three operators beside those of `perf/operators.py`:

  rms_norm   rows plus the block's output so far, divided by their root mean square; the result in the rows' type
             or in 8 bits (e4m3) with a scale for each row, which the gated pair reads; and the gradient
  gated      act(x Wg) * (x Wu), in 16 or 32 bits or of 8-bit rows and weights with scales; and the gradient, which forms x Wg and x Wu anew
  adamw      one step of AdamW over all tensors of a head, moments in 32 or in 8 bits

Row counts are those of the engine's results (one node, the nodes that a batch changed, all nodes of a graph), widths the layer widths
of `synth.workloads` (64, 100, 128, 256, 602), the gated width 8/3 or 4 times that, classes 41, 47, 172 or a list of up to 100 000 items.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-6
TOP = 448.0                                                      # the largest e4m3 number
BLOCK = 128                                                      # elements of a tensor that share a scale of their 8-bit moments
BETA1, BETA2, ADAM_EPS, DECAY, RATE = 0.9, 0.999, 1e-8, 0.01, 3e-4


def _rms(name, rows, cols, type, residual=False, out=None, back=False):
    """back with residual: a gradient arrives at the sum as well as at the normalised rows."""
    return dict(name=name, op="rms_norm", rows=rows, cols=cols, type=type, residual=residual, out=out or type, back=back)


def _gated(name, rows, cols, hidden, type, act="silu", out=None, back=False):
    return dict(name=name, op="gated", rows=rows, cols=cols, hidden=hidden, type=type, act=act, out=out or type, back=back)


def _adamw(name, width, hidden, blocks, classes, type, grad, copy=None, bits=32, step=1000):
    """type: of the parameters, grad: of the gradients, copy: of the copy that the products read, if there is one."""
    return dict(name=name, op="adamw", width=width, hidden=hidden, blocks=blocks, classes=classes, type=type, grad=grad, copy=copy, bits=bits,
                step=step)


def listed():
    return [
        # one new node on its way through a block: latency alone
        _rms("rms-f32-1x128-res", 1, 128, "f32", residual=True),
        # all nodes of a graph of 2.45M, hidden width 256
        _rms("rms-bf16-2.45Mx256-res", 2_450_000, 256, "bf16", residual=True),
        # 8-bit rows for the gated pair, 602 features: rows that start nowhere round
        _rms("rms-e4m3-1Mx602-res", 1_000_000, 602, "bf16", residual=True, out="e4m3"),
        # the gradient in a training step over all nodes
        _rms("rms-grad-bf16-2.45Mx128-res", 2_450_000, 128, "bf16", residual=True, back=True),
        # one node through the pair: the weights are what is read
        _gated("gated-bf16-1x256x683", 1, 256, 683, "bf16"),
        # the nodes that a large batch changed, in full precision
        _gated("gated-f32-50kx128x344", 50_000, 128, 344, "f32", act="gelu"),
        # all nodes of the graph, a width that memory and the matrix units feel alike
        _gated("gated-bf16-2.45Mx128x344", 2_450_000, 128, 344, "bf16"),
        # 8-bit rows and weights, four times the width
        _gated("gated-e4m3-612kx256x1024", 612_500, 256, 1024, "e4m3", act="gelu", out="bf16"),
        # the gradient of a training step over 233k nodes
        _gated("gated-grad-bf16-233kx256x683", 233_000, 256, 683, "bf16", back=True),
        # a small head: six tensors, latency
        _adamw("adamw-f32-128x344x47", 128, 344, 1, 47, "f32", "f32"),
        # a head that ranks a long list, moments in 8 bits, 16-bit gradients and copy
        _adamw("adamw-8bit-256x683-4-100k", 256, 683, 4, 100_003, "f32", "bf16", copy="bf16", bits=8),
        # a deep head: 64 blocks of three matrices and a norm each, moments in 32 bits
        _adamw("adamw-f32-602x1605-64", 602, 1605, 64, 41, "f32", "bf16", copy="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms_norm", "gated", "gated", "adamw"])
    if op == "adamw":
        width = rng.choice([_log_uniform(rng, 16, 1024), 64, 100, 128, 256, 602])
        type = rng.choice(["f32", "f32", "bf16"])
        c = _adamw("", width, rng.choice([width * 8 // 3, width * 4, _log_uniform(rng, 16, 4096)]), _log_uniform(rng, 1, 64),
                   rng.choice([_log_uniform(rng, 7, 100_000), 41, 47, 172]), type, rng.choice(["f32", "bf16", "f16"]),
                   rng.choice([None, "bf16", "f16"]) if type == "f32" else None, rng.choice([32, 8, 8]), _log_uniform(rng, 1, 100_000))
    else:
        type = rng.choice(["f32", "bf16", "bf16", "f16"])
        back = rng.random() < 0.4
        rows = _log_uniform(rng, 1, 2_450_000)
        if op == "rms_norm":
            out = "e4m3" if not back and rng.random() < 0.4 else type
            c = _rms("", rows, rng.choice([_log_uniform(rng, 16, 4096), 64, 100, 128, 256, 602]), type, rng.random() < 0.7, out, back)
        else:
            cols = rng.choice([_log_uniform(rng, 16, 1024), 64, 100, 128, 256, 602])
            hidden = rng.choice([cols * 8 // 3, cols * 4, _log_uniform(rng, 16, 4096)])
            act = rng.choice(["silu", "gelu", "relu", "none"])
            if not back and rng.random() < 0.35:
                c = _gated("", rows, cols, hidden, "e4m3", act, rng.choice(["f32", "bf16", "f16"]))
            else:
                c = _gated("", rows, cols, hidden, type, act, None, back)
    most = [work(x) for x in listed() if x["op"] == op]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    if c["op"] == "gated" and "f32" in c["type"]:
        most["flops"] /= 8                                       # the matrix units are that much slower in 32 bits
    over = max(work(c)[k] / most[k] for k in most)
    if over > 1:
        if op == "adamw":
            c["blocks"], c["classes"] = max(1, int(c["blocks"] / over)), max(7, int(c["classes"] / over))
        else:
            c["rows"] = max(1, int(c["rows"] / over))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------- inputs
def _shapes(case):
    """The tensors of a head: blocks of norm, gate, up and down, then a norm and a classifier with its bias."""
    w, h, c = case["width"], case["hidden"], case["classes"]
    return [(w,), (w, h), (w, h), (h, w)] * case["blocks"] + [(w,), (w, c), (c,)]


def _starts(case):
    """Where the tensors start in one buffer that holds them all, on multiples of BLOCK, and its length."""
    starts, at = [], 0
    for shape in _shapes(case):
        starts.append(at)
        at += -(-math.prod(shape) // BLOCK) * BLOCK
    return starts, at


def _views(case, flat):
    starts = _starts(case)[0]
    return [flat[s:s + math.prod(shape)].view(shape) for s, shape in zip(starts, _shapes(case))]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    s = dict(case)
    if case["op"] == "adamw":
        _prepare_adamw(case, seed, randn, s)
        return s
    rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
    if case["op"] == "rms_norm":
        # a residual stream: the scale of a row differs from node to node
        x = randn(rows, cols).mul_(randn(rows, 1).mul_(0.5).exp_())
        s.update(x=x.to(t), weight=(1 + 0.1 * randn(cols)).to(t))
        if case["back"]:
            s["rstd"] = (s["x"].float().square_().mean(1) + EPS).rsqrt()
            s["dy"] = randn(rows, cols).to(t)
            s["d_total"] = randn(rows, cols).to(t) if case["residual"] else None
        else:
            s["res"] = randn(rows, cols).to(t) if case["residual"] else None
        return s
    # normalised rows, and weights whose products have a variance of about 1
    hidden = case["hidden"]
    x, w = randn(rows, cols), randn(2, cols, hidden).mul_(cols ** -0.5)
    if case["type"] == "e4m3":
        scale = x.abs().amax(1) / TOP
        w_scale = w.abs().amax(1) / TOP
        s.update(x=x.div_(scale[:, None]).to(t), x_scale=scale, gate_scale=w_scale[0], up_scale=w_scale[1])
        w = w.div_(w_scale[:, None]).transpose(1, 2).contiguous().to(t)                   # a hidden unit's weights side by side
        s.update(w_gate=w[0].t(), w_up=w[1].t())
    else:
        s.update(x=x.to(t), w_gate=w[0].to(t), w_up=w[1].to(t))
        if case["back"]:
            s["dh"] = randn(rows, hidden).to(t)
    return s


def _prepare_adamw(case, seed, randn, s):
    n = _starts(case)[1]
    here = torch.zeros(n, device="cuda")                         # 1 in the tensors, 0 between them
    for v in _views(case, here):
        v.fill_(1)
    # gradients whose size differs from element to element, and the moments that they leave behind
    size = randn(n).mul_(0.5).exp_().mul_(1e-3).mul_(here)
    grad = randn(n).mul_(size)
    m = randn(n).mul_(0.3).mul_(size)
    root = randn(n).mul_(0.1).add_(1).abs_().mul_(size)          # of the second moment
    s["grad_scale"] = 1.0
    if case["grad"] == "f16":                                    # scaled for the range of half precision
        s["grad_scale"] = 1.0 / 1024
        grad.mul_(1024)
    s.update(param=randn(n).mul_(0.05).mul_(here).to(TYPES[case["type"]]), grad=grad.to(TYPES[case["grad"]]), seed=seed)
    s["copy"] = s["param"].to(TYPES[case["copy"]]) if case["copy"] else None
    if case["bits"] == 8:
        for name, v in (("m", m), ("v", root)):
            scale = v.view(-1, BLOCK).abs().amax(1) / TOP
            s[name] = v.view(-1, BLOCK).div(scale.clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = scale
    else:
        s.update(m=m, v=root.square_())
    # what the step takes: every tensor with its gradient, moments and copy
    s["params"], s["grads"] = _views(case, s["param"]), _views(case, s["grad"])
    s["copies"] = _views(case, s["copy"]) if case["copy"] else None
    if case["bits"] == 8:
        starts = _starts(case)[0]
        shapes = _shapes(case)
        scales = [slice(at // BLOCK, at // BLOCK - (-math.prod(shape) // BLOCK)) for at, shape in zip(starts, shapes)]
        s["moments"] = [(a, s["m_scale"][at], b, s["v_scale"][at]) for a, b, at in zip(_views(case, s["m"]), _views(case, s["v"]), scales)]
    else:
        s["moments"] = list(zip(_views(case, s["m"]), _views(case, s["v"])))


# ---------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return _run_own(s)
    return {"rms_norm": _plain_rms, "gated": _plain_gated, "adamw": _plain_adamw}[s["op"]](s)


def _run_own(s):
    from paper_2309_11071_amd import head
    if s["op"] == "rms_norm":
        if s["back"]:
            return head.rms_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"], d_total=s["d_total"])
        return head.rms_norm(s["x"], s["weight"], residual=s["res"], eps=EPS, out_dtype=TYPES[s["out"]])
    if s["op"] == "gated":
        if s["back"]:
            return head.gated_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], act=s["act"])
        if s["type"] == "e4m3":
            return head.gated(s["x"], s["w_gate"], s["w_up"], act=s["act"], x_scale=s["x_scale"], gate_scale=s["gate_scale"],
                              up_scale=s["up_scale"], out_dtype=TYPES[s["out"]])
        return head.gated(s["x"], s["w_gate"], s["w_up"], act=s["act"])
    head.adamw(s["params"], s["grads"], s["moments"], s["step"], lr=RATE, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
               grad_scale=s["grad_scale"], copies=s["copies"], seed=s["seed"])
    return _adamw_buffers(s)


def _adamw_buffers(s):
    return [s["param"], s["copy"], s["m"], s.get("m_scale"), s["v"], s.get("v_scale")]


def _plain_rms(s):
    t, weight = s["x"].dtype, s["weight"].float()
    if not s["back"]:
        total = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(t)
        x = total.float()
        rstd = (x.square().mean(1) + EPS).rsqrt()
        y = x * rstd[:, None] * weight
        if s["out"] != "e4m3":
            return y.to(t), total, rstd
        scale = y.abs().amax(1) / TOP
        return (y / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.float8_e4m3fn), scale, total, rstd
    rstd = s["rstd"][:, None]
    h, dy = s["x"].float() * rstd, s["dy"].float()
    dweight = (dy * h).sum(0)
    g = dy * weight
    dx = rstd * (g - h * (g * h).mean(1, keepdim=True))
    if s["d_total"] is not None:
        dx = dx + s["d_total"].float()
    return dx.to(t), dweight.to(t)


def _plain_act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_act_grad(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    return torch.ones_like(z)


def _plain_gated(s):
    t, act = TYPES[s["out"]], s["act"]
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg, x @ wu
    if s["type"] == "e4m3":
        g = g * s["x_scale"][:, None] * s["gate_scale"]
        u = u * s["x_scale"][:, None] * s["up_scale"]
    if not s["back"]:
        return (_plain_act(g, act) * u).to(t)
    dh = s["dh"].float()
    dg, du = dh * u * _plain_act_grad(g, act), dh * _plain_act(g, act)
    dx = dg @ wg.t() + du @ wu.t()
    return dx.to(t), (x.t() @ dg).to(t), (x.t() @ du).to(t)


def _mix(x):
    """A 32-bit number of a 32-bit number, all bits of it depending on all bits (multipliers: of the golden ratio and of the root of 3)."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(s):
    """Two random numbers of 32 bits for every element, of seed, step, tensor and element."""
    shapes, (starts, n) = _shapes(s), _starts(s)
    which = torch.zeros(n, dtype=torch.int64, device="cuda")
    which[torch.tensor(starts[1:], device="cuda")] = 1
    which = which.cumsum(0)
    key = torch.zeros(len(shapes), dtype=torch.int64, device="cuda")
    for part in (torch.arange(len(shapes), device="cuda"), s["step"] & 0xFFFFFFFF, s["step"] >> 32, s["seed"] & 0xFFFFFFFF, s["seed"] >> 32 & 0xFFFFFFFF):
        key = _mix((key + part + 0x6A09E667) & 0xFFFFFFFF)
    at = torch.arange(n, device="cuda") - torch.tensor(starts, device="cuda")[which]
    first = _mix((at & 0xFFFFFFFF) ^ _mix((key[which] + (at >> 32)) & 0xFFFFFFFF))
    return first, _mix((first + 0x6A09E667) & 0xFFFFFFFF)


def _plain_to_8_bits(x, random, floor):
    """Codes and scales of blocks; a number between two codes goes to one or the other, the nearer the likelier.  floor: no number but 0 becomes 0."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) / TOP
    a = x.abs() * torch.where(scale > 0, 1 / scale, 0.0)[:, None]
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))) / 8
    step = torch.where(step * 8 > a.clamp(min=2.0 ** -6), step / 2, step)                  # where the logarithm was rounded up
    count = ((a.double() / step * 2 ** 20).long() + (random & 0xFFFFF).view(-1, BLOCK)) >> 20
    q = (count * step).clamp(max=TOP)
    if floor:
        q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q.float(), x).to(torch.float8_e4m3fn).view(-1), scale


def _plain_to_bf16(x, random):
    """float to bfloat16, up or down by chance: the nearer the likelier."""
    bits = x.view(torch.int32).long() & 0xFFFFFFFF
    bits = (bits + (random & 0xFFFF)) >> 16
    return torch.where(bits >= 1 << 15, bits - (1 << 16), bits).to(torch.int16).view(torch.bfloat16)


def _plain_adamw(s):
    eight, t = s["bits"] == 8, s["step"]
    first, second = _random(s) if eight or s["type"] == "bf16" else (None, None)
    p, g = s["param"].float(), s["grad"].float() * s["grad_scale"]
    if eight:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    root = v.sqrt()
    by_m, by_v = RATE / -math.expm1(t * math.log(BETA1)), 1 / math.sqrt(-math.expm1(t * math.log(BETA2)))
    p = p * (1 - RATE * DECAY) - by_m * m / (root * by_v + ADAM_EPS)
    if s["type"] == "bf16":
        s["param"].copy_(_plain_to_bf16(p, (first >> 20) + ((second >> 20 & 15) << 12)))
    else:
        s["param"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if eight:
        codes, scale = _plain_to_8_bits(m, first, False)
        s["m"].copy_(codes), s["m_scale"].copy_(scale)
        codes, scale = _plain_to_8_bits(root, second, True)
        s["v"].copy_(codes), s["v_scale"].copy_(scale)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    return _adamw_buffers(s)


# ---------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rms_norm": _exact_rms, "gated": _exact_gated, "adamw": _exact_adamw}[case["op"]](s)


def _exact_rms(s):
    n, weight = s["x"].shape[1], s["weight"].double()
    if not s["back"]:
        total = s["x"].double()
        if s["res"] is not None:
            total = (total + s["res"].double()).to(s["x"].dtype).double()                  # the sum is defined as it is stored
        rstd = (torch.linalg.vecdot(total, total, dim=1) / n + EPS).pow(-0.5)
        y = torch.einsum("rc,r,c->rc", total, rstd, weight)
        if s["out"] != "e4m3":
            return y, total, rstd
        scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / TOP
        y.mul_(torch.where(scale == 0, scale, scale.reciprocal())[:, None])
        step = torch.ldexp(torch.ones_like(y), (torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
        return torch.round(y / step) * step, scale, total, rstd
    # y_j = x_j r w_j, d r / d x_i = -r^3 x_i / n
    x, r, dy = s["x"].double(), s["rstd"].double()[:, None], s["dy"].double()
    dweight = torch.linalg.vecdot(dy, x * r, dim=0)
    dy.mul_(weight)
    along = torch.linalg.vecdot(dy, x, dim=1)[:, None] / n
    dx = dy.mul_(r).addcmul_(x, along * r.pow(3), value=-1)
    return dx if s["d_total"] is None else dx.add_(s["d_total"].double()), dweight


def _exact_gated(s):
    x, wg, wu = s["x"].double(), s["w_gate"].double(), s["w_up"].double()
    if s["type"] == "e4m3":
        x = x * s["x_scale"].double()[:, None]
        wg, wu = wg * s["gate_scale"].double(), wu * s["up_scale"].double()
    g, u = torch.mm(x, wg), torch.mm(x, wu)
    cdf = {"relu": lambda: (g > 0).double(), "gelu": lambda: torch.special.ndtr(g), "silu": lambda: torch.sigmoid(g), "none": lambda: torch.ones_like(g)}[s["act"]]()
    if not s["back"]:
        return g.mul_(cdf).mul_(u)
    dh = s["dh"].double()
    du = dh * g * cdf
    slope = cdf                                                  # act(z) = z F(z): its slope is F + z F'
    if s["act"] == "gelu":
        slope = cdf + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
    elif s["act"] == "silu":
        slope = cdf + g * cdf * torch.sigmoid(-g)
    dg = dh.mul_(u).mul_(slope)
    return torch.addmm(torch.mm(dg, wg.t()), du, wu.t()), torch.mm(x.t(), dg), torch.mm(x.t(), du)


def _exact_adamw(s):
    n, eight = s["param"].numel(), s["bits"] == 8
    g = s["grad"].double().mul_(s["grad_scale"])
    spread = (lambda scale: scale.double().repeat_interleave(BLOCK)) if eight else None
    m = s["m"].double() * spread(s["m_scale"]) if eight else s["m"].double()
    v = (s["v"].double() * spread(s["v_scale"])).pow(2) if eight else s["v"].double()
    m.lerp_(g, 1 - BETA1)
    v.lerp_(g.square(), 1 - BETA2)
    unbiased = (v / (1 - BETA2 ** s["step"])).sqrt_().add_(ADAM_EPS)
    p = s["param"].double()
    p -= RATE * (DECAY * p + m / (1 - BETA1 ** s["step"]) / unbiased)
    copy = p if s["copy"] is not None else None
    if not eight and s["type"] != "bf16":
        return [p, copy, m, None, v, None]

    def scrambled(z):
        for shift, by in ((16, 0x9E3779B1), (15, 0xBB67AE85)):
            z = (z ^ z >> shift) * by & 0xFFFFFFFF
        return z ^ z >> 16
    index, key = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
    for k, (start, shape) in enumerate(zip(_starts(s)[0], _shapes(s))):
        end = start - (-math.prod(shape) // BLOCK) * BLOCK
        z = 0
        for part in (k, s["step"] % 2 ** 32, s["step"] // 2 ** 32, s["seed"] % 2 ** 32, s["seed"] // 2 ** 32 % 2 ** 32):
            z = scrambled(z + part + 0x6A09E667 & 0xFFFFFFFF)
        index[start:end] = torch.arange(end - start, device="cuda")
        key[start:end] = scrambled(z)                            # every tensor has fewer than 2^32 elements here
    chance = scrambled(index ^ key)
    other = scrambled(chance + 0x6A09E667 & 0xFFFFFFFF)

    def by_chance(a, step, bits, numbers):
        """a's magnitude to a multiple of step: down, or up where the number of that many bits and the rest pass one."""
        count = torch.floor(torch.floor(a.abs() / step * 2 ** bits).add_(numbers).mul_(2.0 ** -bits))
        return torch.copysign(count * step, a)

    def power(a, least):
        return torch.ldexp(torch.ones_like(a), (torch.frexp(a).exponent - 1).clamp(min=least))
    if s["type"] == "bf16":
        p = by_chance(p, power(p, -126) / 128, 16, chance // 2 ** 20 + other // 2 ** 20 % 16 * 2 ** 12)
    if not eight:
        return [p, copy, m, None, v, None]
    out = []
    for a, numbers, least in ((m, chance, 0.0), (v.sqrt(), other, 2.0 ** -9)):
        scale = torch.linalg.vector_norm(a.view(-1, BLOCK), ord=math.inf, dim=1) / TOP
        a = a * torch.where(scale == 0, scale, scale.reciprocal()).repeat_interleave(BLOCK)
        q = by_chance(a, power(a, -6) / 8, 20, numbers % 2 ** 20).clamp(-TOP, TOP)
        out += [torch.where((a > 0) & (q < least), least, q) if least else q, scale]
    return [p, copy] + out


# ---------------------------------------------------------------------------------------- what it takes
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    if case["op"] == "adamw":
        n = float(sum(math.prod(shape) for shape in _shapes(case)))
        moments = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        e = 2 * SIZE[case["type"]] + SIZE[case["grad"]] + (SIZE[case["copy"]] if case["copy"] else 0) + moments
        return {"bytes": e * n, "flops": 14.0 * n}
    r, c, e = float(case["rows"]), case["cols"], SIZE[case["type"]]
    if case["op"] == "rms_norm":
        if case["back"]:                                         # dy, total, d_total -> dx; rstd; weight -> dweight
            return {"bytes": e * r * c * (3 + case["residual"]) + 4 * r + 2.0 * e * c, "flops": 9.0 * r * c}
        out = SIZE[case["out"]] * r * c + (4 * r if case["out"] == "e4m3" else 0)
        return {"bytes": e * r * c * (1 + 2 * case["residual"]) + out + 4 * r + e * c, "flops": 5.0 * r * c}
    h = case["hidden"]
    if case["back"]:                                             # dh, x, both weights -> dx and the weights' gradients
        return {"bytes": e * (r * h + 2 * r * c + 4.0 * c * h), "flops": 12.0 * r * c * h}
    scales = 4 * r + 8.0 * h if case["type"] == "e4m3" else 0
    return {"bytes": e * (r * c + 2.0 * c * h) + SIZE[case["out"]] * r * h + scales, "flops": 4.0 * r * c * h}
