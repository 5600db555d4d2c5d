"""References in 64 bits for the operators of include/zf_layer.h, and storage
helpers.  Nothing here uses the library."""
import numpy as np
import torch

F64 = torch.float64


def e4m3(v):
    """v (float64) rounded to the nearest e4m3 value, ties to even; |v| <= 448."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=-6) - 3)
    return torch.round(v / step) * step


def group_max(x, group):
    r, c = x.shape
    big = torch.zeros(-(-r // group) * group, -(-c // 128) * 128, dtype=F64)
    big[:r, :c] = x.abs()
    return big.view(-1, group, big.shape[1] // 128, 128).amax((1, 3))


def quantize(x, group):
    """(element values, codes) of x (float64, CPU)."""
    r, c = x.shape
    top = group_max(torch.where(x.isnan(), float("inf"), x), group)
    bad = torch.isinf(top)
    codes = torch.arange(0, 248, dtype=F64)
    limit = 448.0 * 2.0 ** (codes - 127.0)
    code = torch.searchsorted(limit, torch.where(bad, 0.0, top))  # limit[code - 1] < top <= limit[code]
    code = torch.where(bad, 255, code)
    per = code.repeat_interleave(group, 0)[:r].repeat_interleave(128, 1)[:, :c]
    q = e4m3(torch.where(per == 255, 0.0, x) * 2.0 ** (127.0 - per.to(F64)))
    return q, code.to(torch.uint8)


def value(q, code, group):
    """What elements and codes stand for (float64)."""
    r, c = q.shape
    s = torch.where(code == 255, float("nan"), 2.0 ** (code.to(F64) - 127.0))
    return q.to(F64) * s.repeat_interleave(group, 0)[:r].repeat_interleave(128, 1)[:, :c]


def fp8_buffers(zf, rows, cols, group, fill_data=0x7F, fill_scale=0xFF, extra=16):
    """An Fp8 inside larger buffers whose other bytes are `fill` (a NaN each),
    and the buffers."""
    sr, sc = -(-rows // group), -(-cols // 128)
    ld, lds = -(-cols // 16) * 16 + extra, -(-sc // 4) * 4 + 4
    data = torch.full((rows + 1, ld), fill_data, dtype=torch.uint8, device="cuda")
    scale = torch.full((sr + 1, lds), fill_scale, dtype=torch.uint8, device="cuda")
    f = zf.Fp8(data.view(torch.float8_e4m3fn)[:rows, :cols],
               scale.view(torch.float8_e8m0fnu)[:sr, :sc], group)
    return f, data, scale


def random_fp8(zf, rows, cols, group, gen, spread=3):
    """An operand of random finite elements and scales, everything around it NaN;
    and the values it stands for."""
    f, data, scale = fp8_buffers(zf, rows, cols, group)
    sr, sc = f.scale.shape
    b = torch.randint(0, 256, (rows, cols), generator=gen, dtype=torch.uint8)
    b = torch.where((b & 0x7F) == 0x7F, b - 1, b)
    code = (127 - spread + torch.randint(0, 2 * spread + 1, (sr, sc), generator=gen)).to(torch.uint8)
    data[:rows, :cols] = b.cuda()
    scale[:sr, :sc] = code.cuda()
    return f, value(b.view(torch.float8_e4m3fn), code, group)


def strided(t, pad, offset=0):
    """t on the GPU as rows of a wider buffer that starts `offset` elements in."""
    r, c = t.shape
    buf = torch.full((r * (c + pad) + offset + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[offset:offset + r * (c + pad)].view(r, c + pad)[:, :c]
    v.copy_(t)
    return v


# ---- AdamW in numpy, one fp32 operation at a time ------------------------------

def f32(x):
    return np.float32(x)


def np_e4m3(x):
    """fp32 array -> e4m3 codes (uint8); NaN -> 0x7f."""
    t = torch.from_numpy(np.nan_to_num(x.astype(np.float64), nan=0.0))
    v = e4m3(t).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
    v[np.isnan(x)] = 0x7F
    return v


def np_decode(codes, scale):
    v = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    return v * np.repeat(scale, 128)[:v.size]


def np_encode(x, second):
    n = x.size
    big = np.zeros(-(-n // 128) * 128, np.float32)
    big[:n] = np.sqrt(x) if second else x
    big = big.reshape(-1, 128)
    bits = np.abs(big).view(np.uint32).max(1, keepdims=True)
    top = bits.view(np.float32)
    small = top < f32(2.0 ** -100)
    inv = np.where(small, f32(0), f32(448) / np.where(small, f32(1), top))
    codes = np_e4m3(big * inv)
    if second:
        keep = (codes == 0) & (big > 0) & ~small & (inv > 0)
        codes = np.where(keep, np.uint8(1), codes)
    scale = np.where(small, f32(0), top / f32(448)).reshape(-1)
    return codes.reshape(-1)[:n].astype(np.uint8), scale


def np_adamw(g, p, m, v, lr, b1, b2, eps, wd, step, gs=None):
    """One step; fp32 arrays in, (p, m, v) out."""
    c = [f32(x) for x in (b1, 1 - b1, b2, 1 - b2, lr, eps, lr * wd, 1 / (1 - b1 ** step),
                          1 / (1 - b2 ** step))]
    B1, C1, B2, C2, LR, EPS, WD, IB1, IB2 = c
    with np.errstate(all="ignore"):
        if gs is not None:
            g = g * f32(gs)
        m = B1 * m + C1 * g
        v = B2 * v + C2 * (g * g)
        u = (m * IB1) / (np.sqrt(v * IB2) + EPS)
        if WD != 0:
            p = p - WD * p
        return p - LR * u, m, v
