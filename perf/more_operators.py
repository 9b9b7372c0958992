"""What is measured of a student's further operators: the label loss over the LM head, the gated linear layer, the layer norm
and rotary positions. `run` computes an operator with elementary torch operations in 32 bits where `own` is false, and
through this package where it is true; `exact` computes the same from the definitions in 64 bits."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GROUP = 32                                   # values of a row that share one power of two in an 8-bit record
IGNORED = -100
EPS = 1e-5


def listed():
    return [
        # queries and keys of one generated token, far into a long context
        dict(name="rotary_1x40x128_forward", op="rotary", T=1, heads=32, kv=8, D=128, R=128, layout="half", type="bf16",
             scaling="none", far=100000, train=False),
        # a short packed batch, part of each head rotated in interleaved pairs, positions interpolated
        dict(name="rotary_2047x24x96_train", op="rotary", T=2047, heads=16, kv=8, D=96, R=64, layout="interleaved",
             type="f16", scaling="linear", far=8192, train=True),
        # a 32K-token sequence of a student whose context was extended
        dict(name="rotary_32768x40x128_train", op="rotary", T=32768, heads=32, kv=8, D=128, R=128, layout="half",
             type="bf16", scaling="yarn", far=32768, train=True),
        # one generated token: forward only, nothing kept
        dict(name="norm_1x4096_forward", op="norm", T=1, H=4096, type="bf16", weight="bf16", bias=True, train=False),
        # a short ragged batch, without bias, its weight kept in fp32
        dict(name="norm_1021x2880_train", op="norm", T=1021, H=2880, type="bf16", weight="f32", bias=False, train=True),
        # a 32K-token sequence
        dict(name="norm_32768x4096_train", op="norm", T=32768, H=4096, type="bf16", weight="bf16", bias=True, train=True),
        # the feed-forward block's first half for one generated token
        dict(name="gated_1x2048x5632_forward", op="gated", T=1, H=2048, F=5632, act="silu", format="none", train=False),
        # a short ragged batch; gate and up are computed again in the backward pass
        dict(name="gated_1021x2816x7168_train", op="gated", T=1021, H=2816, F=7168, act="gelu", format="none", train=True),
        # a 16K-token sequence; gate, up and the input are kept in 8 bits
        dict(name="gated_16384x2048x5632_train", op="gated", T=16384, H=2048, F=5632, act="silu", format="int8", train=True),
        # an evaluation batch's losses, token by token
        dict(name="label_333x2816x32768_eval", op="label", T=333, H=2816, V=32768, smoothing=0.0, z=0.0, weighted=False,
             train=False),
        # a short batch over an odd vocabulary, with smoothing, a z term and weighted tokens
        dict(name="label_1021x2880x20001_train", op="label", T=1021, H=2880, V=20001, smoothing=0.1, z=1e-4, weighted=True,
             train=True),
        # two chunks of a step over a large vocabulary
        dict(name="label_8192x2048x131072_train", op="label", T=8192, H=2048, V=131072, smoothing=0.0, z=0.0,
             weighted=False, train=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rotary", "norm", "gated", "label"])
    if op == "rotary":
        D = rng.choice([64, 80, 96, 128, 192, 256])
        kv = rng.choice([1, 2, 4, 8, 12])
        heads = kv * rng.choice([1, 2, 4, 5])
        most = min(32768, 32768 * 40 * 128 // ((heads + kv) * D))
        return dict(op=op, T=_spread(rng, 1, most), heads=heads, kv=kv, D=D, R=rng.choice([D, D, D // 2]),
                    layout=rng.choice(["half", "interleaved"]), type=rng.choice(["bf16", "bf16", "f16", "f32"]) if most < 32768
                    else rng.choice(["bf16", "f16"]), scaling=rng.choice(["none", "linear", "ntk", "yarn"]),
                    far=_spread(rng, 2048, 1000000), train=rng.random() < 0.7)
    if op == "norm":
        H = 8 * _spread(rng, 32, 1024) + (rng.randrange(1, 8) if rng.random() < 0.2 else 0)
        return dict(op=op, T=_spread(rng, 1, 32768 * 4096 // max(H, 4096)), H=H, type=rng.choice(["bf16", "bf16", "f16"]),
                    weight=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.7, train=rng.random() < 0.8)
    if op == "gated":
        H, F = 8 * _spread(rng, 32, 352), 8 * _spread(rng, 64, 896)
        return dict(op=op, T=_spread(rng, 1, min(16384, 16384 * 2048 * 5632 // (H * F))), H=H, F=F,
                    act=rng.choice(["silu", "gelu"]), format=rng.choice(["none", "int8", "e4m3"]), train=rng.random() < 0.8)
    H, V = 8 * _spread(rng, 32, 512), _spread(rng, 1000, 131072)
    smooth = rng.random() < 0.4
    return dict(op=op, T=_spread(rng, 1, min(8192, 8192 * 2048 * 131072 // (H * V))), H=H, V=V,
                smoothing=rng.choice([0.05, 0.1]) if smooth else 0.0, z=rng.choice([0.0, 0.0, 1e-4]),
                weighted=rng.random() < 0.3, train=rng.random() < 0.7)


def work(case):
    """Inputs read once and outputs written once, by each pass; a record that a training step keeps between its two
    passes is written once and read once."""
    T = case["T"]
    if case["op"] == "rotary":
        n = T * (case["heads"] + case["kv"]) * case["D"] * (2 if case["train"] else 1)
        return {"bytes": n * 2 * BYTES[case["type"]], "flops": 3 * n}
    if case["op"] == "norm":
        n = T * case["H"]
        return {"bytes": n * BYTES[case["type"]] * (5 if case["train"] else 2), "flops": n * (20 if case["train"] else 7)}
    if case["op"] == "gated":
        H, F = case["H"], case["F"]
        forward = 2 * T * H + 4 * H * F + 2 * T * F
        if not case["train"]:
            return {"bytes": forward, "flops": 4 * T * H * F}
        kept = 4 * T * F * (1 + 1 / GROUP) if case["format"] != "none" else 0
        x = T * H * (2 if case["format"] == "none" else 1 + 1 / GROUP)
        return {"bytes": forward + kept + 2 * T * F + x + 4 * H * F + 2 * T * H + 4 * H * F, "flops": 12 * T * H * F}
    H, V = case["H"], case["V"]
    if not case["train"]:
        return {"bytes": 2 * T * H + 2 * V * H + 12 * T, "flops": 2 * T * H * V}
    return {"bytes": 4 * T * H + 4 * V * H + 12 * T, "flops": 6 * T * H * V}


# ------------------------------------------------------------------ inputs


def _positions(g, T, far):
    """Packed documents: positions run up, and start again at a few places; somewhere below `far`."""
    starts = torch.rand(T, generator=g, device="cuda") < 4 / max(T, 4)
    starts[0] = True
    steps = torch.arange(T, device="cuda")
    base = torch.where(starts, steps, torch.zeros_like(steps)).cummax(0).values
    first = torch.randint(0, max(1, far - T), (1,), generator=g, device="cuda")
    return steps - base + first


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    T, s = case["T"], {"case": case}
    if case["op"] == "rotary":
        kind, D, q, k = TYPES[case["type"]], case["D"], case["heads"], case["kv"]
        qkv = normal(T, q + 2 * k, D).to(kind)                              # one projection's queries, keys and values
        s["q"], s["k"], s["positions"] = qkv[:, :q], qkv[:, q:q + k], _positions(g, T, case["far"])
        if case["train"]:
            s["dq"], s["dk"] = (0.01 * normal(T, q, D)).to(kind), (0.01 * normal(T, k, D)).to(kind)
        if own:
            from paper_2608_03796_b200 import body
            s["layer"] = body.Rotary(D, rotary_dim=case["R"], layout=case["layout"], **_rope(case))
    elif case["op"] == "norm":
        H, kind, wide = case["H"], TYPES[case["type"]], TYPES[case["weight"]]
        x = normal(T, H) * torch.exp(0.5 * normal(H)) + 0.3 * normal(H)     # channels of their own width and centre
        s["x"] = x.to(kind)
        s["weight"] = (1 + 0.2 * normal(H)).to(wide)
        s["bias"] = (0.1 * normal(H)).to(wide) if case["bias"] else None
        if case["train"]:
            s["dy"] = (0.01 * normal(T, H)).to(kind)
        if own:
            from paper_2608_03796_b200 import body
            s["layer"] = body.LayerNorm(T, H, dtype=kind, eps=EPS, train=case["train"])
    elif case["op"] == "gated":
        H, F = case["H"], case["F"]
        s["x"] = normal(T, H).bfloat16()                                    # a normed hidden state
        s["weight"] = (1.5 * normal(2 * F, H) / H ** 0.5).bfloat16()
        if case["train"]:
            s["dh"] = (0.01 * normal(T, F)).bfloat16()
        form = None if case["format"] == "none" else case["format"]
        if own:
            from paper_2608_03796_b200 import body
            s["layer"] = body.GatedLinear(T, H, F, act=case["act"], act8=form, train=case["train"])
            s["record"] = body.Act8Record(T, H, form).store(s["x"]) if case["train"] and form else None
        elif case["train"] and form:
            s["kept_x"] = _as_recorded(s["x"].float(), form)                # what the norm before this layer left behind
    else:
        H, V = case["H"], case["V"]
        s["hidden"] = (1.5 * normal(T, H)).bfloat16()
        s["weight"] = (normal(V, H) / H ** 0.5).bfloat16()
        s["labels"] = torch.randint(0, V, (T,), generator=g, device="cuda")
        skipped = torch.rand(T, generator=g, device="cuda") < 0.1           # prompts and padding
        skipped[T - T // 16:] = True
        s["labels"][skipped] = IGNORED
        s["token_weight"] = 2 * torch.rand(T, generator=g, device="cuda") if case["weighted"] else None
        if own:
            from paper_2608_03796_b200 import labels
            s["layer"] = labels.LabelLoss(T, H, V, label_smoothing=case["smoothing"], z_loss=case["z"],
                                          ignore_index=IGNORED, train=case["train"])
    return s


def _rope(case):
    kind = case["scaling"]
    return dict(base=10000.0, scaling=kind, factor=1.0 if kind == "none" else 4.0, original_length=4096)


# ------------------------------------------------------------------ one pass


def run(s):
    case = s["case"]
    if own:
        return _own(case, s)
    if case["op"] == "rotary":
        cos, sin, scale = _angles(case, s["positions"])
        out = [_turn(case, x, cos * scale, sin * scale) for x in (s["q"], s["k"])]
        if case["train"]:
            out += [_turn(case, x, cos * scale, -sin * scale) for x in (s["dq"], s["dk"])]
        return out
    if case["op"] == "norm":
        return _norm(s["x"], s["weight"], s["bias"], s.get("dy"))
    if case["op"] == "gated":
        return _gated(case, s)
    return _label(case, s)


def _own(case, s):
    layer = s["layer"]
    if case["op"] == "rotary":
        out = list(layer.forward(s["q"], s["k"], s["positions"]))
        return out + list(layer.backward(s["dq"], s["dk"], s["positions"])) if case["train"] else out
    if case["op"] == "norm":
        y = layer.forward(s["x"], s["weight"], s["bias"])
        if not case["train"]:
            return [y]
        d = layer.backward(s["dy"])
        return [y, d.x, d.weight] + ([d.bias] if case["bias"] else [])
    if case["op"] == "gated":
        h = layer.forward(s["x"], s["weight"])
        return [h, *layer.backward(s["dh"], record=s["record"])] if case["train"] else [h]
    if case["train"]:
        return list(layer.step(s["hidden"], s["weight"], s["labels"], token_weight=s["token_weight"]))
    loss = layer.forward(s["hidden"], s["weight"], s["labels"], token_weight=s["token_weight"])
    return [loss, layer.losses]


def _frequencies(case):
    """Radians a position, of each pair, and what the rotated values are multiplied by."""
    r, R = _rope(case), case["R"]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    base, factor = r["base"], r["factor"]
    if case["scaling"] == "ntk":
        base = base * factor ** (R / (R - 2))
    f = base ** (-2 * i / R)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "yarn":
        turns = r["original_length"] * f / (2 * math.pi)                    # over the length that was trained on
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        f = (1 - keep) * f / factor + keep * f
        return f, 1 + 0.1 * math.log(factor)
    return f, 1.0


def _angles(case, positions):
    f, scale = _frequencies(case)
    a = positions.double()[:, None] * f                                     # far positions: 32 bits would lose the angle
    return a.cos().float()[:, None], a.sin().float()[:, None], scale


def _turn(case, x, cos, sin):
    R = case["R"]
    x32 = x.float()
    if case["layout"] == "half":
        a, b = x32[..., :R // 2], x32[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x32[..., 0:R:2], x32[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x32[..., R:]], dim=-1).to(x.dtype)


def _norm(x, weight, bias, dy):
    x32, w = x.float(), weight.float()
    centred = x32 - x32.mean(1, keepdim=True)
    rho = 1 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xh = centred * rho
    y = xh * w if bias is None else xh * w + bias.float()
    if dy is None:
        return [y.to(x.dtype)]
    d = dy.float()
    dxh = d * w
    dx = rho * (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True))
    out = [y.to(x.dtype), dx.to(x.dtype), (d * xh).sum(0, dtype=torch.float64).to(weight.dtype)]
    return out if bias is None else out + [d.sum(0, dtype=torch.float64).to(bias.dtype)]


def _act(act, x):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p * (1 + x * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)


def _as_recorded(x, form):
    """The values that an 8-bit record of x [T, W] stands for."""
    T, W = x.shape
    rows = torch.nn.functional.pad(x, (0, -W % GROUP)).reshape(T, -1, GROUP)
    most = 127.0 if form == "int8" else 448.0
    part, e = torch.frexp(rows.abs().amax(-1, keepdim=True) / most)
    e = torch.where(part == 0.5, e - 1, e).clamp(min=-126)                  # smallest e with max <= most 2^e
    codes = torch.ldexp(rows, -e)
    codes = torch.round(codes) if form == "int8" else codes.to(torch.float8_e4m3fn).to(x.dtype)
    return torch.ldexp(codes, e).reshape(T, -1)[:, :W]


def _gated(case, s):
    F, x, w = case["F"], s["x"].float(), s["weight"].float()
    z = x @ w.t()
    gate, up = z[:, :F], z[:, F:]
    h = (_act(case["act"], gate)[0] * up).bfloat16()
    if not case["train"]:
        return [h]
    if case["format"] != "none":
        gate, up, x = _as_recorded(gate, case["format"]), _as_recorded(up, case["format"]), s["kept_x"]
    a, da = _act(case["act"], gate)
    dh = s["dh"].float()
    dz = torch.cat([dh * up * da, dh * a], dim=1)
    return [h, (dz @ w).bfloat16(), (dz.t() @ x).bfloat16()]


def _label(case, s):
    h, w, labels, V = s["hidden"].float(), s["weight"].float(), s["labels"], case["V"]
    counted = labels != IGNORED
    y = torch.where(counted, labels, torch.zeros_like(labels))
    z = h @ w.t()
    top = z.max(1).values
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    smooth, lam = case["smoothing"], case["z"]
    losses = lse - (1 - smooth) * z.gather(1, y[:, None])[:, 0] - smooth * z.mean(1) + lam * lse * lse
    losses = torch.where(counted, losses, torch.zeros_like(losses))
    n = counted.sum().clamp(min=1)
    share = counted.float() / n if s["token_weight"] is None else counted * s["token_weight"] / n
    loss = (losses.double() * share).sum().float().reshape(1)
    if not case["train"]:
        return [loss, losses]
    z.sub_(lse[:, None]).exp_().mul_((1 + 2 * lam * lse)[:, None]).sub_(smooth / V)
    z.scatter_add_(1, y[:, None], torch.full_like(z[:, :1], smooth - 1))
    z.mul_(share[:, None])
    return [loss, (z @ w).bfloat16(), (z.t() @ h).bfloat16()]


# ------------------------------------------------------------------ 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    with torch.enable_grad():
        return {"rotary": _exact_rotary, "norm": _exact_norm, "gated": _exact_gated, "label": _exact_label}[case["op"]](case, s)


def _exact_rotary(case, s):
    R, r = case["R"], _rope(case)
    L, S, scale, freq = r["original_length"], r["factor"], 1.0, []
    for i in range(R // 2):
        f = r["base"] ** (-2.0 * i / R)
        if case["scaling"] == "linear":
            f /= S
        elif case["scaling"] == "ntk":
            f = (r["base"] * S ** (R / (R - 2.0))) ** (-2.0 * i / R)
        elif case["scaling"] == "yarn":
            ramp = min(1.0, max(0.0, (L * f / (2 * math.pi) - 1.0) / 31.0))
            f = f / S * (1 - ramp) + f * ramp
            scale = 0.1 * math.log(S) + 1
        freq.append(f)
    angle = s["positions"].double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")

    def turned(x, way):
        y = x.double()
        pairs = y[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2) if case["layout"] == "half" \
            else y[..., :R].unflatten(-1, (R // 2, 2))
        z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angle, scale), way * angle)
        z = torch.view_as_real(z)
        z = z.transpose(-1, -2) if case["layout"] == "half" else z
        return torch.cat([z.flatten(-2), y[..., R:]], dim=-1)
    out = [turned(s["q"], 1), turned(s["k"], 1)]
    return out + [turned(s["dq"], -1), turned(s["dk"], -1)] if case["train"] else out


def _exact_norm(case, s):
    x, w = s["x"].double().requires_grad_(), s["weight"].double().requires_grad_()
    b = None if s["bias"] is None else s["bias"].double().requires_grad_()
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    y = (x - mean) * (var + EPS) ** -0.5 * w + (0 if b is None else b)
    if not case["train"]:
        return [y.detach()]
    return [y.detach(), *torch.autograd.grad(y, [x, w] if b is None else [x, w, b], s["dy"].double())]


def _exact_act(act, x):
    return x * torch.sigmoid(x) if act == "silu" else x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def _exact_record(x, form):
    T, W = x.shape
    rows = torch.nn.functional.pad(x, (0, -W % GROUP)).reshape(-1, GROUP)
    most = 127.0 if form == "int8" else 448.0
    step = torch.exp2(torch.ceil(torch.log2(rows.abs().amax(1).clamp(min=most * 2.0 ** -126) / most)))[:, None]
    codes = rows / step
    if form == "int8":
        codes = codes.round()
    else:                                                                   # 3 bits behind the leading one, 2^-9 at least
        ulp = torch.exp2(torch.floor(torch.log2(codes.abs().clamp(min=2.0 ** -6))) - 3)
        codes = (codes / ulp).round() * ulp
    return (codes * step).reshape(T, -1)[:, :W]


def _exact_gated(case, s):
    F, x = case["F"], s["x"].double()
    wg, wu = s["weight"][:F].double(), s["weight"][F:].double()
    gate, up = x @ wg.t(), x @ wu.t()
    h = _exact_act(case["act"], gate) * up
    if not case["train"]:
        return [h]
    if case["format"] != "none":
        gate, up, x = (_exact_record(v, case["format"]) for v in (gate, up, x))
    gate.requires_grad_(), up.requires_grad_()
    dgate, dup = torch.autograd.grad(_exact_act(case["act"], gate) * up, (gate, up), s["dh"].double())
    return [h, dgate @ wg + dup @ wu, torch.cat([dgate.t() @ x, dup.t() @ x])]


def _exact_label(case, s):
    h, w = s["hidden"].double().requires_grad_(), s["weight"].double().requires_grad_()
    counted = s["labels"] != IGNORED
    logp = torch.log_softmax(h @ w.t(), dim=1)
    lse = -logp[:, 0] + (h @ w[0])
    hard = logp.gather(1, s["labels"].clamp(min=0)[:, None])[:, 0]
    losses = -(1 - case["smoothing"]) * hard - case["smoothing"] * logp.mean(1) + case["z"] * lse ** 2
    losses = losses * counted
    each = losses if s["token_weight"] is None else losses * s["token_weight"].double()
    loss = each.sum() / max(1, int(counted.sum()))
    if not case["train"]:
        return [loss.detach().reshape(1), losses.detach()]
    return [loss.detach().reshape(1), *torch.autograd.grad(loss, (h, w))]
