"""8-bit codes of a cache's rows on the CPU, written from their definition (test infrastructure)."""
import torch

CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}


def scale64(top, code):
    """The smallest power of two, from 2^-100 on, with top <= LARGEST times it; NaN for rows that are not finite."""
    s = torch.full_like(top, 2.0 ** -100)
    for _ in range(260):
        s = torch.where(top > LARGEST[code] * s, 2 * s, s)
    return torch.where(torch.isfinite(top), s, torch.nan)


def step64(v, code):
    """Distance of neighbouring codes at v (in units of the scale)."""
    if code == "int8":
        return torch.ones_like(v)
    return torch.exp2((torch.frexp(v).exponent - 1).clamp(min=-6).double() - 3)


def decode64(code, scale, kind):
    """Values of codes (uint8 bits) and scales, from the bits."""
    c = code.to(torch.int64)
    if kind == "int8":
        v = (c - 256 * (c >= 128)).double()
    else:
        e, f = (c >> 3) & 15, (c & 7).double()
        v = torch.where(e == 0, f / 512, (8 + f) * torch.exp2(e.double() - 10))
        v = torch.where((c & 127) == 127, torch.nan, v)
        v = torch.where(c >= 128, -v, v)
    return v * scale.double()[..., None]


def quantise64(x, kind):
    """Codes (uint8 bits), scales (fp64) and values of rows x [..., 64]: rounded to nearest, ties to even."""
    x = x.double()
    s = scale64(x.abs().amax(dim=-1), kind)
    odd = ~torch.isfinite(s)
    v = torch.where(odd[..., None], 0.0, x / s[..., None])
    # the largest code whose value is below 2^128: values past it would not be numbers in fp32
    most = torch.where(s == (2.0 ** 122 if kind == "int8" else 2.0 ** 120), 63.0 if kind == "int8" else 240.0, 1e9)
    v = torch.minimum(torch.maximum(v, -most[..., None]), most[..., None])
    if kind == "int8":
        code = (torch.round(v).to(torch.int64) & 255).to(torch.uint8)
    else:
        step = step64(v, kind)
        r = torch.round(v / step) * step
        a = r.abs()
        e = torch.frexp(a).exponent - 1
        normal = e >= -6
        bits = torch.where(normal, ((e + 7) << 3) + ((a / torch.exp2(e.double()) - 1) * 8).to(torch.int64),
                           (a * 512).to(torch.int64))
        code = (torch.where(a == 0, torch.zeros_like(bits), bits) + 128 * torch.signbit(v)).to(torch.uint8)
    return code, s, decode64(code, s, kind)
