"""The operators of the layer around an updated weight, as they are measured.

Four operators: the RMS norm with the residual's addition and an 8-bit output,
the quantiser to 8-bit floating point, the matrix product of 8-bit operands
with a scale for each 128 elements, and the AdamW step over many tensors with
states in 32 or 8 bits.  Each has a plain form in elementary torch operations
(32 bits, rounded once at the end) and, where `own` is set, the library's call.

The 8-bit format: e4m3 elements, e8m0 scales (2^(code - 127)), the least code
with which a group's largest magnitude fits 448; 255 where the group holds an
infinity or a NaN.  Groups are 128 consecutive elements of a row (group 1) or
128 x 128 blocks (group 128).

A case is a dict of plain values:
  kind    "norm", "norm_backward", "quantize", "matmul", "linear", "adamw";
  rows, cols     tokens and width ("norm*", "quantize", "linear": cols = in);
  n              outputs ("matmul", "linear"); k the reduction ("matmul");
  dtype          "bf16" or "f32" of the activations, or of the output ("matmul");
  out            what a norm returns: "y", "q" or "yq";
  residual       whether the norm adds one (backward: takes the gradient of one);
  group          rows that share a scale: the quantiser's, the product's second operand's;
  copies         "rows", "transposed" or "both" ("quantize");
  pad            extra elements between rows (views of wider buffers);
  sizes          elements of each tensor ("adamw"), "count*size" terms;
  bits           32 or 8, the states' ("adamw"); grad "bf16" or "f32"; decay.
"""

import math

import torch

own = False

EPS = 1e-6
LR, BETA1, BETA2, ADAM_EPS = 1e-5, 0.9, 0.999, 1e-8
LAYER_7B = "4*16777216 3*45088768"  # the seven linear weights of one Llama-2-7B layer


def listed():
    return [
        # Serving: one token of a 4096-wide model, residual added, the 8-bit
        # operand of the next product written.  Latency is its cost.
        dict(name="norm-token", kind="norm", rows=1, cols=4096, dtype="bf16", out="q",
             residual=True, pad=0),
        # Training: a batch of 8192 tokens; both the bf16 rows (kept for the
        # backward pass) and the 8-bit operand.
        dict(name="norm-8192x4096", kind="norm", rows=8192, cols=4096, dtype="bf16", out="yq",
             residual=True, pad=0),
        # Odd sizes in 32 bits, rows inside a wider buffer.
        dict(name="norm-backward-odd-f32", kind="norm_backward", rows=1237, cols=5003, dtype="f32",
             residual=False, pad=5),
        # The same norm's gradients, with the residual stream's gradient added.
        dict(name="norm-backward-8192x4096", kind="norm_backward", rows=8192, cols=4096,
             dtype="bf16", residual=True, pad=0),
        # A gradient on its way to both products of a backward pass.
        dict(name="quantize-both-4096x11008", kind="quantize", rows=4096, cols=11008,
             dtype="bf16", group=1, copies="both", pad=0),
        # Updated weights laid out for the forward and the backward product.
        dict(name="quantize-weight-4099x5003", kind="quantize", rows=4099, cols=5003,
             dtype="bf16", group=128, copies="both", pad=0),
        # Serving one token: the weight is read once, nothing else counts.
        dict(name="matmul-token", kind="matmul", rows=1, n=11008, k=4096, dtype="bf16", group=128),
        # A prompt of 2048 tokens through the down projection.
        dict(name="matmul-prompt", kind="matmul", rows=2048, n=4096, k=11008, dtype="bf16",
             group=128),
        # Odd sizes in every direction, 32-bit output (logits of a pruned model).
        dict(name="matmul-odd-f32", kind="matmul", rows=1003, n=5003, k=3001, dtype="f32",
             group=1),
        # Training: a linear layer's forward and backward pass, quantising
        # included, the weight gradient stored channel-major.
        dict(name="linear-8192", kind="linear", rows=8192, cols=4096, n=11008),
        # The norm gains of a 32-layer model: many small tensors, one launch.
        dict(name="adamw-gains", kind="adamw", sizes="65*4096", bits=32, grad="f32", decay=0.0),
        # The weights of one 7B layer with states in 8 bits.
        dict(name="adamw-layer-8bit", kind="adamw", sizes=LAYER_7B, bits=8, grad="bf16",
             decay=0.01),
    ]


# ---- drawn cases ------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Any integer between lo and hi, or a multiple of 64 as layers mostly have."""
    x = _log(rng, lo, hi)
    if rng.random() < 0.55 and hi >= 64:
        x = max(64, 64 * (x // 64))
    return x + 64 if x == 3072 else x


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "quantize", "matmul", "matmul", "linear", "adamw",
                       "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 8, 3])
    if kind == "norm":
        return dict(kind=kind, rows=_size(rng, 1, 8192), cols=_size(rng, 128, 8192), dtype=dtype,
                    out=rng.choice(["y", "q", "yq"]), residual=rng.random() < 0.7, pad=pad)
    if kind == "norm_backward":
        return dict(kind=kind, rows=_size(rng, 16, 8192), cols=_size(rng, 128, 8192), dtype=dtype,
                    residual=rng.random() < 0.7, pad=pad)
    if kind == "quantize":
        return dict(kind=kind, rows=_size(rng, 1, 8192), cols=_size(rng, 128, 8192), dtype=dtype,
                    group=rng.choice([1, 1, 128]), copies=rng.choice(["rows", "transposed", "both"]),
                    pad=pad)
    if kind == "matmul":
        rows = _size(rng, 1, 64) if rng.random() < 0.5 else _size(rng, 64, 8192)
        return dict(kind=kind, rows=rows, n=_size(rng, 128, 11008), k=_size(rng, 128, 11008),
                    dtype=dtype, group=rng.choice([1, 128]))
    if kind == "linear":
        return dict(kind=kind, rows=_size(rng, 64, 8192), cols=_size(rng, 256, 4096),
                    n=_size(rng, 256, 11008))
    terms = ["%d*%d" % (rng.randint(1, 64), _size(rng, 1, 16384))]
    if rng.random() < 0.7:
        terms.append("%d*%d" % (rng.randint(1, 4), _size(rng, 65536, 33554432)))
    return dict(kind=kind, sizes=" ".join(terms), bits=rng.choice([8, 32]),
                grad=rng.choice(["bf16", "bf16", "f32"]), decay=rng.choice([0.0, 0.01]))


# ---- inputs -----------------------------------------------------------------

def _torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(gen, rows, cols, dtype, pad=0, std=1.0):
    """Normal elements in rows of cols + pad."""
    buf = torch.randn(rows, cols + pad, generator=gen, device="cuda") * std
    return buf.to(dtype)[:, :cols]


def _activations(gen, rows, cols, dtype, pad=0):
    """Activations as a decoder layer has them: normal, with a scale per
    channel of which a few are large."""
    scale = torch.exp(torch.randn(cols + pad, generator=gen, device="cuda"))
    buf = torch.randn(rows, cols + pad, generator=gen, device="cuda")
    return (buf * scale).to(dtype)[:, :cols]


def _padded(t, unit):
    """`t` as a view of rows whose length is a multiple of `unit`."""
    rows, cols = t.shape
    buf = torch.zeros(rows, -(-cols // unit) * unit, dtype=t.dtype, device=t.device)
    buf[:, :cols] = t
    return buf[:, :cols]


def _operand(gen, rows, cols, group, std):
    """An 8-bit operand a program keeps: elements in rows of a multiple of 16
    bytes, scales in rows of a multiple of 4."""
    q, code = _plain_quantize(_normal(gen, rows, cols, torch.float32, std=std), group)
    q = _padded(q.view(torch.uint8), 16).view(torch.float8_e4m3fn)
    return q, _padded(code, 4).view(torch.float8_e8m0fnu)


def _sizes(case):
    out = []
    for term in case["sizes"].split():
        count, size = term.split("*")
        out += [int(size)] * int(count)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind in ("norm", "norm_backward"):
        dt, rows, cols = _torch_dtype(case["dtype"]), case["rows"], case["cols"]
        s["x"] = _activations(gen, rows, cols, dt, case["pad"])
        s["gain"] = (1.0 + 0.1 * torch.randn(cols, generator=gen, device="cuda")).to(dt)
        if case["residual"]:
            s["residual"] = _activations(gen, rows, cols, dt, case["pad"])
        if kind == "norm_backward":
            s["dy"] = _normal(gen, rows, cols, dt, case["pad"], std=0.01)
            h = s["x"].float()
            s["rstd"] = 1.0 / torch.sqrt((h * h).mean(-1) + EPS)
    elif kind == "quantize":
        s["x"] = _activations(gen, case["rows"], case["cols"], _torch_dtype(case["dtype"]),
                              case["pad"])
    elif kind == "matmul":
        s["a"] = _operand(gen, case["rows"], case["k"], 1, 1.0)
        s["b"] = _operand(gen, case["n"], case["k"], case["group"], 0.02)
    elif kind == "linear":
        rows, cols, n = case["rows"], case["cols"], case["n"]
        s["x"] = _activations(gen, rows, cols, torch.bfloat16)
        s["dy"] = _normal(gen, rows, n, torch.bfloat16, std=0.01)
        s["w"] = _operand(gen, n, cols, 128, 0.02)
        # the same weight laid out for the backward product
        q, scale = s["w"]
        s["wt"] = (_padded(q.view(torch.uint8).t(), 16).view(torch.float8_e4m3fn),
                   _padded(scale.view(torch.uint8).t(), 4).view(torch.float8_e8m0fnu))
    else:
        sizes, gdt = _sizes(case), _torch_dtype(case["grad"])

        def rand(n, std):
            return torch.randn(n, generator=gen, device="cuda") * std

        s["grad"] = [rand(n, 1e-3).to(gdt) for n in sizes]
        s["master"] = [rand(n, 0.02) for n in sizes]
        s["weight"] = [p.to(torch.bfloat16) for p in s["master"]]
        m, v = [rand(n, 1e-4) for n in sizes], [rand(n, 1e-3).square() for n in sizes]
        if case["bits"] == 8:
            m, v = [_plain_encode(t, False) for t in m], [_plain_encode(t, True) for t in v]
        s["exp_avg"], s["exp_avg_sq"], s["step"] = m, v, 100
        s["grad_scale"] = torch.full((1,), 0.5, device="cuda")  # a clipped step
    return s


# ---- the plain forms ----------------------------------------------------------

def _groups(x, group):
    """x [r, c] padded with zeros, as [R, group, C, 128]."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % group))
    return x.view(x.shape[0] // group, group, x.shape[1] // 128, 128)


def _plain_quantize(x, group):
    """(e4m3 elements [r, c], e8m0 codes [ceil(r / group), ceil(c / 128)])"""
    r, c = x.shape
    g = _groups(x.float(), group)
    bits = g.abs().amax(3).amax(1).view(torch.int32)
    code = torch.where(bits >= 0x7F800000, 255, ((bits + 0x1FFFFF) >> 23).sub(8).clamp(min=0))
    mult = ((254 - code).clamp(min=0) << 23).view(torch.float32)[:, None, :, None]
    q = torch.where(code[:, None, :, None] == 255, 0.0, g * mult)
    q = q.reshape(g.shape[0] * group, -1)[:r, :c].to(torch.float8_e4m3fn)
    return q, code.to(torch.uint8)


def _plain_dequantize(operand, group):
    q, scale = operand
    s = (scale.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)
    s = torch.where(scale.view(torch.uint8) == 0, 2.0 ** -127, s)
    s = s.repeat_interleave(128, 1)[:, :q.shape[1]].repeat_interleave(group, 0)[:q.shape[0]]
    return q.float() * s


def _plain_norm(s):
    c, x = s["case"], s["x"]
    h = (x.float() + s["residual"].float()).to(x.dtype) if c["residual"] else x
    hf = h.float()
    rstd = 1.0 / torch.sqrt((hf * hf).mean(-1) + EPS)
    y = (hf * rstd[:, None] * s["gain"].float()).to(x.dtype)
    out = {"rstd": rstd}
    if c["residual"]:
        out["h"] = h
    if "y" in c["out"]:
        out["y"] = y
    if "q" in c["out"]:
        q, code = _plain_quantize(y, 1)
        out["q"], out["scale"] = q, code.view(torch.float8_e8m0fnu)
    return out


def _plain_norm_backward(s):
    x = s["x"].float()
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    hh = x * rstd
    t = dy * s["gain"].float()
    dx = rstd * (t - hh * (t * hh).mean(-1, keepdim=True))
    if s["case"]["residual"]:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(s["x"].dtype), "dgain": (dy * hh).sum(0)}


def _plain_quantize_case(s):
    c, x, out = s["case"], s["x"], {}
    if c["copies"] != "transposed":
        q, code = _plain_quantize(x, c["group"])
        out["q"], out["scale"] = q, code.view(torch.float8_e8m0fnu)
    if c["copies"] != "rows":
        q, code = _plain_quantize(x.t(), c["group"])
        out["qt"], out["scale_t"] = q, code.view(torch.float8_e8m0fnu)
    return out


def _plain_matmul(a, b, group_b, dtype):
    return (_plain_dequantize(a, 1) @ _plain_dequantize(b, group_b).t()).to(dtype)


def _plain_operand(x):
    q, code = _plain_quantize(x, 1)
    return q, code.view(torch.float8_e8m0fnu)


def _plain_linear(s):
    x, dy, bf16 = s["x"], s["dy"], torch.bfloat16
    return {"y": _plain_matmul(_plain_operand(x), s["w"], 128, bf16),
            "dx": _plain_matmul(_plain_operand(dy), s["wt"], 128, bf16),
            "dw": _plain_matmul(_plain_operand(x.t()), _plain_operand(dy.t()), 1, bf16)}


def _plain_encode(t, second):
    """A state in 8 bits: (e4m3 codes [n], fp32 scales [ceil(n / 128)]) of the
    first moment, or of the second moment's square root."""
    n = t.numel()
    x = torch.nn.functional.pad(torch.sqrt(t) if second else t, (0, -n % 128)).view(-1, 128)
    top = x.abs().amax(1, keepdim=True)
    small, limit = top < 2.0 ** -100, torch.full_like(top, 448.0)
    inv = torch.where(small, 0.0, limit / top)
    q = (x * inv).to(torch.float8_e4m3fn)
    if second:  # what is not zero stays so
        code = q.view(torch.uint8)
        code = torch.where((code == 0) & (x > 0) & ~small, 1, code).to(torch.uint8)
        q = code.view(torch.float8_e4m3fn)
    return q.view(-1)[:n], torch.where(small, 0.0, top / limit).view(-1)


def _plain_decode(state, second):
    q, scale = state
    x = q.float() * scale.repeat_interleave(128)[:q.numel()]
    return x * x if second else x


def _f32(x):
    return torch.tensor(x, dtype=torch.float64).to(torch.float32).item()


def _plain_adamw_tensor(g, p, w, m, v, scale, step, decay, bits):
    """One tensor's step; the state's own tensors are updated."""
    b1, c1, b2, c2 = _f32(BETA1), _f32(1.0 - BETA1), _f32(BETA2), _f32(1.0 - BETA2)
    ib1, ib2 = _f32(1.0 / (1.0 - BETA1 ** step)), _f32(1.0 / (1.0 - BETA2 ** step))
    g = g.float() * scale
    m1 = _plain_decode(m, False) if bits == 8 else m
    v1 = _plain_decode(v, True) if bits == 8 else v
    m1 = b1 * m1 + c1 * g
    v1 = b2 * v1 + c2 * (g * g)
    u = (m1 * ib1) / (torch.sqrt(v1 * ib2) + _f32(ADAM_EPS))
    p1 = p - _f32(LR * decay) * p if decay else p
    p.copy_(p1 - _f32(LR) * u)
    w.copy_(p)
    if bits == 8:
        (mq, ms), (vq, vs) = _plain_encode(m1, False), _plain_encode(v1, True)
        m[0].copy_(mq), m[1].copy_(ms), v[0].copy_(vq), v[1].copy_(vs)
    else:
        m.copy_(m1), v.copy_(v1)


def _cat(tensors):
    return torch.cat([t.view(torch.uint8) for t in tensors]).view(torch.float8_e4m3fn) \
        if tensors[0].dtype == torch.float8_e4m3fn else torch.cat(tensors)


def _adamw_outputs(s):
    """Every tensor's new values, the tensors joined end to end."""
    out = {"master": s["master"], "weight": s["weight"]}
    if s["case"]["bits"] == 8:
        out["exp_avg"], out["exp_avg_scale"] = zip(*s["exp_avg"])
        out["exp_avg_sq"], out["exp_avg_sq_scale"] = zip(*s["exp_avg_sq"])
    else:
        out["exp_avg"], out["exp_avg_sq"] = s["exp_avg"], s["exp_avg_sq"]
    # a few tensors are returned as they are, many of them joined
    if len(s["master"]) <= 8:
        return {k: list(v) for k, v in out.items()}
    return {k: _cat(list(v)) for k, v in out.items()}


def _plain_adamw(s):
    c = s["case"]
    s["step"] += 1
    [_plain_adamw_tensor(g, p, w, m, v, s["grad_scale"], s["step"], c["decay"], c["bits"])
     for g, p, w, m, v in zip(s["grad"], s["master"], s["weight"], s["exp_avg"], s["exp_avg_sq"])]
    return _adamw_outputs(s)


# ---- the library's calls --------------------------------------------------------

def _own_norm(s, zf):
    c = s["case"]
    r = zf.rmsnorm(s["x"], s["gain"], residual=s.get("residual"), eps=EPS, want_y="y" in c["out"],
                   want_q="q" in c["out"])
    out = {"rstd": r.rstd}
    if c["residual"]:
        out["h"] = r.h
    if "y" in c["out"]:
        out["y"] = r.y
    if "q" in c["out"]:
        out["q"], out["scale"] = r.q.data, r.q.scale
    return out


def _own_norm_backward(s, zf):
    dx, dgain = zf.rmsnorm_backward(s["dy"], s["x"], s["gain"], s["rstd"],
                                    dresidual=s.get("residual"))
    return {"dx": dx, "dgain": dgain}


def _own_quantize(s, zf):
    c, out = s["case"], {}
    q, qt = zf.quantize_fp8(s["x"], group=c["group"], rows=c["copies"] != "transposed",
                            transposed=c["copies"] != "rows")
    if q is not None:
        out["q"], out["scale"] = q.data, q.scale
    if qt is not None:
        out["qt"], out["scale_t"] = qt.data, qt.scale
    return out


def _own_matmul(s, zf):
    c = s["case"]
    return {"out": zf.matmul_fp8(zf.Fp8(*s["a"], 1), zf.Fp8(*s["b"], c["group"]),
                                 dtype=_torch_dtype(c["dtype"]))}


def _own_linear(s, zf):
    x, xt = zf.quantize_fp8(s["x"], transposed=True)
    dy, dyt = zf.quantize_fp8(s["dy"], transposed=True)
    return {"y": zf.matmul_fp8(x, zf.Fp8(*s["w"], 128)),
            "dx": zf.matmul_fp8(dy, zf.Fp8(*s["wt"], 128)),
            "dw": zf.matmul_fp8(xt, dyt)}


def _own_adamw(s, zf):
    c = s["case"]
    if "plan" not in s:  # as a program makes it before its first step
        s["plan"] = zf.AdamWPlan([
            zf.AdamWBuffers(g, p, *((m[0], v[0]) if c["bits"] == 8 else (m, v)), weight=w,
                            exp_avg_scale=m[1] if c["bits"] == 8 else None,
                            exp_avg_sq_scale=v[1] if c["bits"] == 8 else None)
            for g, p, w, m, v in zip(s["grad"], s["master"], s["weight"], s["exp_avg"],
                                     s["exp_avg_sq"])])
        s["hp"] = zf.AdamHparams(LR, BETA1, BETA2, ADAM_EPS, c["decay"])
    s["step"] += 1
    s["plan"].step(s["hp"], s["step"], grad_scale=s["grad_scale"])
    return _adamw_outputs(s)


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2505_12242_amd as zf
        return {"norm": _own_norm, "norm_backward": _own_norm_backward, "quantize": _own_quantize,
                "matmul": _own_matmul, "linear": _own_linear, "adamw": _own_adamw}[kind](state, zf)
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward,
            "quantize": _plain_quantize_case,
            "matmul": lambda s: {"out": _plain_matmul(s["a"], s["b"], s["case"]["group"],
                                                      _torch_dtype(s["case"]["dtype"]))},
            "linear": _plain_linear, "adamw": _plain_adamw}[kind](state)


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    kind = case["kind"]
    e = 4 if case.get("dtype") == "f32" else 2
    if kind in ("norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        if kind == "norm":
            per = e * (1 + 2 * case["residual"] + ("y" in case["out"]))
            per += (1 + 1 / 128) * ("q" in case["out"])
            return {"bytes": per * rows * cols + e * cols + 4 * rows, "flops": 8 * rows * cols}
        per = e * (3 + case["residual"])
        return {"bytes": per * rows * cols + (4 + e) * cols + 4 * rows, "flops": 12 * rows * cols}
    if kind == "quantize":
        rc = case["rows"] * case["cols"]
        copies = 2 if case["copies"] == "both" else 1
        return {"bytes": rc * (e + copies * (1 + 1 / 128)), "flops": 4 * rc * copies}
    if kind == "matmul":
        m, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": (m + n) * k * (1 + 1 / 128) + e * m * n, "flops": 2 * m * n * k}
    if kind == "linear":
        t, i, o = case["rows"], case["cols"], case["n"]
        # x and dy read, y, dx and dw written in bf16; the weight read in two layouts
        return {"bytes": 2 * (2 * t * (i + o) + i * o) + 2 * i * o, "flops": 6 * t * i * o}
    total = sum(_sizes(case))
    per = (4 if case["grad"] == "f32" else 2) + 8 + 2 + (16 if case["bits"] == 32 else 4)
    return {"bytes": per * total, "flops": 20 * total}


# ---- the definitions in 64 bits --------------------------------------------------

_E4M3 = None


def _e4m3_grid():
    """The 127 non-negative e4m3 values in ascending order."""
    global _E4M3
    if _E4M3 is None:
        codes = torch.arange(127, dtype=torch.float64)
        ex, ma = torch.div(codes, 8, rounding_mode="floor"), codes % 8
        _E4M3 = torch.where(ex == 0, ma / 8 * 2.0 ** -6, (1 + ma / 8) * 2.0 ** (ex - 7)).cuda()
    return _E4M3


def _to_e4m3(x):
    """The nearest e4m3 value; ties to the even code.  A slice at a time."""
    grid = _e4m3_grid()
    mid = (grid[1:] + grid[:-1]) / 2
    flat = x.reshape(-1)
    out = torch.empty_like(flat)
    for a in range(0, flat.numel(), 1 << 26):
        v = flat[a:a + (1 << 26)]
        mag = v.abs()
        lo = torch.bucketize(mag, mid, right=False)  # mid[lo - 1] < mag <= mid[lo]
        tie = (lo < 126) & (mag == mid[lo.clamp(max=125)]) & (lo % 2 == 1)
        out[a:a + (1 << 26)] = torch.copysign(grid[(lo + tie.long()).clamp(max=126)], v)
    return out.view_as(x)


def _exact_quantize(x, group):
    """(elements, scales) as numbers, from x in 64 bits."""
    r, c = x.shape
    big = torch.zeros(-(-r // group) * group, -(-c // 128) * 128, dtype=torch.float64,
                      device=x.device)
    big[:r, :c] = x
    top = big.abs().view(-1, group, big.shape[1] // 128, 128).amax((1, 3))
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(448.0 * 2.0 ** e < top, e + 1, e)
    e = torch.where(448.0 * 2.0 ** (e - 1) >= top, e - 1, e).clamp(min=-127.0)
    scale = 2.0 ** e
    spread = scale.repeat_interleave(group, 0).repeat_interleave(128, 1)
    return _to_e4m3((big / spread)[:r, :c]), scale


def _value(operand, group):
    """An operand's elements times their scales in 64 bits."""
    q, scale = operand
    s = 2.0 ** (scale.view(torch.uint8).double() - 127.0)
    rows = torch.arange(q.shape[0], device=q.device) // group
    cols = torch.arange(q.shape[1], device=q.device) // 128
    return q.double() * s[rows][:, cols]


def _rounded(x, dtype):
    return x.to(dtype).double()


def _exact_quantized_value(x):
    q, scale = _exact_quantize(x.double(), 1)
    return q * scale.repeat_interleave(128, 1)[:, :q.shape[1]]


def _exact_state(x, second):
    x = torch.sqrt(x) if second else x
    n = x.numel()
    big = torch.zeros(-(-n // 128) * 128, dtype=torch.float64, device=x.device)
    big[:n] = x
    big = big.view(-1, 128)
    top = big.abs().amax(1, keepdim=True)
    unit = top / 448.0
    q = _to_e4m3(torch.where(top > 0, big / torch.where(top > 0, unit, 1.0), 0.0))
    if second:
        q = torch.where((q == 0) & (big > 0), 2.0 ** -9, q)
    return q.view(-1)[:n], unit.view(-1)


def _exact_adamw(s):
    c = s["case"]
    t = s["step"] + 1
    out = {"master": [], "weight": [], "exp_avg": [], "exp_avg_sq": []}
    if c["bits"] == 8:
        out.update(exp_avg_scale=[], exp_avg_sq_scale=[])
    for i, g in enumerate(s["grad"]):
        g = g.double() * s["grad_scale"].double()
        m, v = s["exp_avg"][i], s["exp_avg_sq"][i]
        if c["bits"] == 8:
            m = m[0].double() * m[1].double().repeat_interleave(128)[:g.numel()]
            v = (v[0].double() * v[1].double().repeat_interleave(128)[:g.numel()]).square()
        m = BETA1 * m.double() + (1 - BETA1) * g
        v = BETA2 * v.double() + (1 - BETA2) * g.square()
        p = s["master"][i].double()
        p = p * (1 - LR * c["decay"])
        p = p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
        out["master"].append(p)
        out["weight"].append(p)
        if c["bits"] == 8:
            for name, x, second in (("exp_avg", m, False), ("exp_avg_sq", v, True)):
                q, unit = _exact_state(x, second)
                out[name].append(q)
                out[name + "_scale"].append(unit)
        else:
            out["exp_avg"].append(m)
            out["exp_avg_sq"].append(v)
    if len(s["grad"]) <= 8:
        return out
    return {k: torch.cat(v) for k, v in out.items()}


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_adamw(s)
    if kind == "matmul":
        return {"out": _value(s["a"], 1) @ _value(s["b"], case["group"]).t()}
    if kind == "linear":
        x, dy = s["x"], s["dy"]
        out = {"y": _exact_quantized_value(x) @ _value(s["w"], 128).t()}
        out["dx"] = _exact_quantized_value(dy) @ _value(s["wt"], 128).t()
        out["dw"] = _exact_quantized_value(x.t()) @ _exact_quantized_value(dy.t()).t()
        return out
    if kind == "quantize":
        out, x = {}, s["x"].double()
        if case["copies"] != "transposed":
            out["q"], out["scale"] = _exact_quantize(x, case["group"])
        if case["copies"] != "rows":
            out["qt"], out["scale_t"] = _exact_quantize(x.t(), case["group"])
        return out
    x, gain, dt = s["x"].double(), s["gain"].double(), s["x"].dtype
    if kind == "norm":
        h = _rounded(x + s["residual"].double(), dt) if case["residual"] else x
        rstd = (h.square().mean(-1) + EPS) ** -0.5
        y = h * rstd[:, None] * gain
        out = {"rstd": rstd}
        if case["residual"]:
            out["h"] = h
        if "y" in case["out"]:
            out["y"] = y
        if "q" in case["out"]:  # what is quantised is the output in its own type
            out["q"], out["scale"] = _exact_quantize(_rounded(y, dt), 1)
        return out
    dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
    hh, cols = x * rstd, x.shape[1]
    dot = (dy * gain * hh).sum(-1, keepdim=True) / cols
    dx = rstd * dy * gain - rstd * hh * dot
    if case["residual"]:
        dx = dx + s["residual"].double()
    return {"dx": dx, "dgain": (dy * hh).sum(0)}
