"""What is measured of the operators for a student's body: 8-bit activation records and the layers that read them
in the backward pass. `run` computes an operator with elementary torch operations in 32 bits where `own` is false, and
through this package where it is true; `exact` computes the same from the definitions in 64 bits."""
import math

import torch

own = False

GROUP = 32                                   # values of a row that share one power of two
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
RECORD = 1 + 1 / GROUP                       # bytes a value that a record holds
EPS = 1e-5


def listed():
    return [
        # one generated token's activations through the record: what a call costs at least
        dict(name="record_1x4096_int8", op="record", T=1, H=4096, type="bf16", format="int8", stride=0),
        # a block of a wider fp32 projection, kept per micro-batch: ragged rows, a row stride
        dict(name="record_2047x2816_f32", op="record", T=2047, H=2816, type="f32", format="int8", stride=2816),
        # the hidden states of a 32K-token sequence between two checkpoints
        dict(name="record_32768x4096_e4m3", op="record", T=32768, H=4096, type="bf16", format="e4m3", stride=0),
        # the gated activation of one generated token: forward only, nothing kept
        dict(name="gated_1x7168_forward", op="gated", T=1, F=7168, act="silu", type="bf16", format="none"),
        # a short micro-batch's feed-forward block, forward and backward
        dict(name="gated_1021x7168_train", op="gated", T=1021, F=7168, act="gelu", type="bf16", format="e4m3"),
        # the feed-forward block of a 32K-token sequence, forward and backward
        dict(name="gated_32768x7168_train", op="gated", T=32768, F=7168, act="silu", type="bf16", format="int8"),
        # a projection's weight gradient for a short ragged batch
        dict(name="dweight_333x2816x2816", op="dweight", T=333, N=2816, H=2816, out="bf16", format="int8"),
        # the same at 4096 tokens for a feed-forward projection, kept in fp32 as a master gradient
        dict(name="dweight_4096x7168x2816_f32", op="dweight", T=4096, N=7168, H=2816, out="f32", format="int8"),
        # a square projection's weight gradient over a 32K-token sequence
        dict(name="dweight_32768x4096x4096", op="dweight", T=32768, N=4096, H=4096, out="bf16", format="e4m3"),
        # one generated token between two blocks: forward only
        dict(name="norm_1x4096_forward", op="norm", T=1, H=4096, gate="none", type="bf16", format="none", train=False),
        # a short ragged batch through a gated block of a student that is being healed
        dict(name="norm_1021x2816_train", op="norm", T=1021, H=2816, gate="token", type="bf16", format="none", train=True),
        # the same between two blocks of a 32K-token sequence, from 8-bit records, with a gate per channel
        dict(name="norm_32768x4096_train", op="norm", T=32768, H=4096, gate="channel", type="bf16", format="int8",
             train=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["record", "gated", "dweight", "norm"])
    T = _spread(rng, 1, 32768)
    # widths of hidden states and projections: mostly multiples of 8 (rows that start on 16 bytes), some odd
    H = 8 * _spread(rng, 32, 512) + (rng.randrange(1, 8) if rng.random() < 0.2 and op != "dweight" else 0)
    form = rng.choice(["int8", "e4m3"])
    if op == "record":
        return dict(op=op, T=T, H=H, type=rng.choice(["bf16", "bf16", "f16", "f32"]), format=form,
                    stride=rng.choice([0, 0, H]))
    if op == "gated":
        return dict(op=op, T=T, F=int(H * rng.choice([1.0, 1.75])), act=rng.choice(["silu", "gelu"]),
                    type=rng.choice(["bf16", "bf16", "f16"]), format=rng.choice([form, form, "none"]))
    if op == "dweight":
        return dict(op=op, T=T, N=8 * _spread(rng, 32, 512), H=H, out=rng.choice(["bf16", "f32"]), format=form)
    return dict(op=op, T=T, H=H, gate=rng.choice(["none", "channel", "token"]), type=rng.choice(["bf16", "bf16", "f16"]),
                format=rng.choice([form, "none"]), train=rng.random() < 0.8)


def work(case):
    """Inputs read once and outputs written once; a record that a training step keeps between its two passes is
    written once and read once (the step is there to keep that and nothing wider)."""
    T = case["T"]
    if case["op"] == "record":
        n = T * case["H"]
        return {"bytes": n * (2 * BYTES[case["type"]] + 2 * RECORD), "flops": 4 * n}
    if case["op"] == "gated":
        n = T * case["F"]
        if case["format"] == "none":
            return {"bytes": 6 * n, "flops": 8 * n}
        return {"bytes": n * (6 + 4 * RECORD + 6), "flops": 30 * n}
    if case["op"] == "dweight":
        N, H = case["N"], case["H"]
        return {"bytes": 2 * T * N + RECORD * T * H + BYTES[case["out"]] * N * H, "flops": 2 * T * N * H}
    n = T * case["H"]
    if not case["train"]:
        return {"bytes": 8 * n, "flops": 12 * n}
    # forward: residual and branch in, sum and normed sum out; backward: two gradients in, two out, and the two kept
    # tensors (the sum is an output already and is read again; the branch is an input that is read again)
    kept = 4 * RECORD if case["format"] != "none" else 4
    return {"bytes": n * (8 + 8 + kept), "flops": 50 * n}


# ------------------------------------------------------------------ inputs


def _activations(g, T, H, outliers=True):
    """Normal values, some channels of them far wider than the rest, as hidden states have them."""
    x = torch.randn(T, H, generator=g, device="cuda")
    if outliers:
        x *= torch.exp(0.5 * torch.randn(H, generator=g, device="cuda"))
        x[:, torch.randint(0, H, (max(1, H // 512),), generator=g, device="cuda")] *= 20.0
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, s = case["T"], {"case": case}
    if case["op"] == "record":
        H, kind = case["H"], TYPES[case["type"]]
        s["x"] = _activations(g, T, H + case["stride"]).to(kind)[:, :H]
    elif case["op"] == "gated":
        F, kind = case["F"], TYPES[case["type"]]
        gate_up = (1.5 * _activations(g, T, 2 * F, False)).to(kind)         # one projection's two halves
        s["gate"], s["up"] = gate_up[:, :F], gate_up[:, F:]
        if case["format"] != "none":
            s["dh"] = (0.01 * _activations(g, T, F, False)).to(kind)
    elif case["op"] == "dweight":
        s["x"] = _activations(g, T, case["H"]).bfloat16()
        s["dy"] = (0.01 * _activations(g, T, case["N"], False)).bfloat16()
    else:
        H, kind = case["H"], TYPES[case["type"]]
        s["residual"] = _activations(g, T, H).to(kind)
        s["branch"] = _activations(g, T, H, False).to(kind)
        s["post"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(kind)
        s["pre"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(kind)
        wide = {"none": 0, "channel": H, "token": T}[case["gate"]]
        s["gate"] = (0.5 + 0.2 * torch.randn(wide, generator=g, device="cuda")).to(kind) if wide else None
        if case["train"]:
            s["dy"] = (0.01 * _activations(g, T, H, False)).to(kind)
            s["dsum"] = (0.01 * _activations(g, T, H, False)).to(kind)
    if own:
        _handles(case, s)
    if case["op"] == "dweight":
        if own:
            s["record"].store(s["x"])                                       # what the forward pass left behind
        else:
            s["codes"], s["exponents"] = _encode(s["x"].float(), case["format"])
        del s["x"]
    return s


def _handles(case, s):
    from paper_2608_03796_b200 import body
    T, form = case["T"], None if case["format"] == "none" else case["format"]
    if case["op"] == "record":
        s["record"] = body.Act8Record(T, case["H"], form)
        s["out"] = torch.empty(T, case["H"], dtype=TYPES[case["type"]], device="cuda")
    elif case["op"] == "gated":
        s["layer"] = body.GatedAct(T, case["F"], act=case["act"], act8=form, dtype=TYPES[case["type"]])
    elif case["op"] == "dweight":
        s["record"] = body.Act8Record(T, case["H"], form)
        s["layer"] = body.Act8WeightGrad(T, case["N"], case["H"], dtype=TYPES[case["out"]])
    else:
        s["layer"] = body.BlockNorm(T, case["H"], dtype=TYPES[case["type"]], gate=case["gate"], act8=form, eps=EPS,
                                    branch_scale=0.75, residual_scale=0.9, train=case["train"])


# ------------------------------------------------------------------ one pass


def run(s):
    case = s["case"]
    if case["op"] == "record":
        if own:
            return s["record"].store(s["x"]).load(s["out"])
        return _decode(*_encode(s["x"].float(), case["format"]), case["H"]).to(s["x"].dtype)
    if case["op"] == "gated":
        if own:
            h = s["layer"].forward(s["gate"], s["up"])
            return [h, *s["layer"].backward(s["dh"])] if "dh" in s else [h]
        return _gated(s)
    if case["op"] == "dweight":
        if own:
            return s["layer"].run(s["dy"], s["record"])
        x = _decode(s["codes"], s["exponents"], case["H"])
        return (s["dy"].float().t() @ x).to(TYPES[case["out"]])
    if own:
        y, total = s["layer"].forward(s["residual"], s["branch"], post_weight=s["post"], pre_weight=s["pre"], gate=s["gate"])
        if not case["train"]:
            return [y, total]
        d = s["layer"].backward(s["dy"], s["dsum"])
        return [y, total, d.residual, d.branch, d.post_weight, d.pre_weight, d.gate]
    return _norm(s)


def _encode(x, form):
    """Codes [T, groups, 32] (fp32 whole numbers, or e4m3 values) and exponents [T, groups, 1] of a record."""
    T, H = x.shape
    pad = -H % GROUP
    if pad:
        x = torch.cat([x, x.new_zeros(T, pad)], 1)
    x = x.reshape(T, -1, GROUP)
    part, e = torch.frexp(x.abs().amax(2, keepdim=True))
    if form == "int8":                                    # the largest code is 127 = 0.9921875 * 2^7
        e = torch.where(part <= 0.9921875, e - 7, e - 6).clamp(min=-126)
        return torch.round(torch.ldexp(x, -e)), e
    e = torch.where(part <= 0.875, e - 9, e - 8).clamp(min=-126)            # 448 = 0.875 * 2^9
    return torch.ldexp(x, -e).to(torch.float8_e4m3fn).float(), e


def _decode(codes, e, H):
    return torch.ldexp(codes, e).reshape(codes.shape[0], -1)[:, :H]


def _through(x, form):
    return _decode(*_encode(x, form), x.shape[1])


def _squash(g, act):
    """act(g) = g * sigmoid(k(g)): that sigmoid and k'."""
    if act == "silu":
        return torch.sigmoid(g), torch.ones_like(g)
    c = 2 * math.sqrt(2 / math.pi)
    return torch.sigmoid(c * (g + 0.044715 * g * g * g)), c * (1 + 3 * 0.044715 * g * g)


def _gated(s):
    case, kind = s["case"], s["gate"].dtype
    g, u = s["gate"].float(), s["up"].float()
    h = (g * _squash(g, case["act"])[0] * u).to(kind)
    if "dh" not in s:
        return [h]
    g, u = _through(g, case["format"]), _through(u, case["format"])
    dh = s["dh"].float()
    p, slope = _squash(g, case["act"])
    return [h, (dh * u * (p + g * p * (1 - p) * slope)).to(kind), (dh * g * p).to(kind)]


def _norm(s):
    case, kind = s["case"], s["branch"].dtype
    alpha, beta = 0.75, 0.9
    b, r = s["branch"].float(), s["residual"].float()
    w1, w2 = s["post"].float(), s["pre"].float()
    gate = 1.0 if s["gate"] is None else s["gate"].float()[:, None] if case["gate"] == "token" else s["gate"].float()
    r1 = torch.rsqrt((b * b).mean(1, keepdim=True) + EPS)
    x = beta * r + alpha * gate * (b * r1 * w1)
    r2 = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    y, total = (x * r2 * w2).to(kind), x.to(kind)
    if not case["train"]:
        return [y, total]
    x = total.float()
    if case["format"] != "none":
        b, x = _through(b, case["format"]), _through(x, case["format"])
    dy, bn, xn = s["dy"].float(), b * r1, x * r2
    gy = dy * w2
    d = s["dsum"].float() + r2 * (gy - xn * (gy * xn).mean(1, keepdim=True))
    dn = alpha * gate * d
    gb = dn * w1
    db = r1 * (gb - bn * (gb * bn).mean(1, keepdim=True))
    dgate = None
    if s["gate"] is not None:
        dgate = (alpha * d * bn * w1).sum(1 if case["gate"] == "token" else 0).to(kind)
    return [y, total, (beta * d).to(kind), db.to(kind), (dn * bn).sum(0).to(kind), (dy * xn).sum(0).to(kind), dgate]


# ------------------------------------------------------------------ the definitions in 64 bits


def _kept64(x, form):
    """What a record of x stands for: within each 32 values of a row, multiples of the smallest power of two (or
    4-bit floating values times it) that the format's largest code still covers the largest of them with."""
    out = torch.empty_like(x)
    top = 127.0 if form == "int8" else 448.0
    for at in range(0, x.shape[1], 4096):                 # in ranges of whole groups: 64-bit copies are large
        v = x[:, at:at + 4096]
        width = v.shape[1]
        v = torch.nn.functional.pad(v, (0, -width % GROUP)).view(x.shape[0], -1, GROUP)
        unit = v.abs().amax(2, keepdim=True) / top
        unit = torch.exp2(torch.ceil(torch.log2(unit)).clamp(min=-126.0))
        short = v.abs().amax(2, keepdim=True) > top * unit                  # where the logarithm was rounded
        spare = v.abs().amax(2, keepdim=True) <= top * unit / 2
        unit = torch.where(short, unit * 2, torch.where(spare & (unit > 2.0 ** -126), unit / 2, unit))
        q = v / unit
        if form == "int8":
            q = torch.round(q)
        else:                                             # 3 mantissa bits above 2^-6, steps of 2^-9 below
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(q / step) * step
        out[:, at:at + 4096] = (q * unit).view(x.shape[0], -1)[:, :width]
    return out


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "record":
        return _kept64(s["x"].double(), case["format"])
    if case["op"] == "gated":
        def act(v):
            if case["act"] == "silu":
                return v / (1 + torch.exp(-v))
            return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))

        g, u = s["gate"].double(), s["up"].double()
        h = act(g) * u
        if "dh" not in s:
            return [h]
        g = _kept64(g, case["format"]).requires_grad_(True)
        u = _kept64(u, case["format"]).requires_grad_(True)
        return [h, *torch.autograd.grad(act(g) * u, (g, u), s["dh"].double())]
    if case["op"] == "dweight":
        g = torch.Generator(device="cuda").manual_seed(seed)                # the activations that prepare() encoded
        x = _activations(g, case["T"], case["H"]).bfloat16().double()
        return s["dy"].double().t() @ _kept64(x, case["format"])
    b, r = s["branch"].double(), s["residual"].double()
    w1, w2 = s["post"].double().requires_grad_(True), s["pre"].double().requires_grad_(True)
    gate = None if s["gate"] is None else s["gate"].double().requires_grad_(True)

    def join(r, b, r1):
        wide = 1.0 if gate is None else gate[:, None] if case["gate"] == "token" else gate
        return 0.9 * r + 0.75 * wide * (b * r1 * w1)

    def inverse_rms(v):
        return 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)

    with torch.no_grad():
        r1 = inverse_rms(b)
        x = join(r, b, r1)
        r2 = inverse_rms(x)
        y = x * r2 * w2
        total = x.clone()
        if not case["train"]:
            return [y, total]
        # the backward pass evaluates the gradient's formula at what was kept of the sum and of the branch
        x = x.to(s["branch"].dtype).double()
        if case["format"] != "none":
            b, x = _kept64(b, case["format"]), _kept64(x, case["format"])
        dy, H = s["dy"].double(), case["H"]
        bn, xn = b * r1, x * r2
        scaled = dy * w2
        d = s["dsum"].double() + r2 * scaled - r2 * xn * ((scaled * xn).sum(1, keepdim=True) / H)
        wide = 1.0 if gate is None else gate[:, None] if case["gate"] == "token" else gate
        into = 0.75 * d * wide
        db = r1 * into * w1 - r1 * bn * ((into * w1 * bn).sum(1, keepdim=True) / H)
        dgate = None
        if gate is not None:
            dgate = (0.75 * d * bn * w1).sum(1 if case["gate"] == "token" else 0)
        return [y, total, 0.9 * d, db, (into * bn).sum(0), (dy * xn).sum(0), dgate]
