"""Plain 64-bit forms of the AdamW step and of its 8-bit states, for the tests.  Independent of the library."""
import math

import torch

BLOCK = 32
LOW = 0xFFFFFFFF
ULP = 2.0 ** -24  # half a step of fp32, relative


def f32(x):
    """A number or a float64 tensor rounded to fp32, still in float64."""
    return x.float().double() if isinstance(x, torch.Tensor) else torch.tensor(x, dtype=torch.float32).double().item()


# ---- the hash that rounds (integers; the low 32 bits of products come out right in int64) -----------------------------


def mix(x):
    x = x & LOW
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & LOW
    x = x ^ (x >> 13)
    x = (x * 0x3C6EF373) & LOW
    return x ^ (x >> 16)


def step_key(seed, step):
    return mix(mix(mix(mix(seed) + (seed >> 32)) + (step & LOW) * 0x9E3779B1) + (step >> 32))


def words(key, place):
    """One number of 32 bits for each place (int64 tensor) of the vector in which tensors follow one another in whole blocks."""
    y = mix((place // 8) * 0x9E3779B1 + key) + (place % 8) * 0x9E3779B1 & LOW
    y = ((y ^ (y >> 15)) * 0xA54FF53B) & LOW
    return y ^ (y >> 16)


# ---- 8 bits ----------------------------------------------------------------------------------------------------------


def in_blocks(x):
    pad = -x.numel() % BLOCK
    return torch.cat([x, x.new_zeros(pad)]).view(-1, BLOCK)


def scales(x):
    """Scale of each block of a float64 tensor of fp32 numbers."""
    most = in_blocks(torch.where(torch.isfinite(x), x.abs(), 0.0)).amax(1)
    return torch.where(most > 0, (torch.frexp(most).exponent - 8 + 127).clamp(min=1), 0).to(torch.uint8)


def each(scale, numel):
    return scale.repeat_interleave(BLOCK)[:numel]


def encode(x, scale, chance, fraction):
    """Codes by the sizes of the steps; ``chance`` in [0, 2^16)."""
    y = torch.where(torch.isfinite(x), x.abs(), 0.0) * 2.0 ** (127.0 - each(scale, x.numel()).double())
    y = torch.where(each(scale, x.numel()) == 0, 0.0, y)
    y = torch.where(y < 2.0 ** -6, f32(y + 2.0 ** -6) - 2.0 ** -6, y)
    exponent = torch.where(y > 0, torch.frexp(y).exponent - 1, -6).clamp(min=-6)
    steps = torch.floor(y * 2.0 ** (fraction - exponent.double()) + (chance.double() + 0.5) / 65536.0).long()
    code = steps + (exponent.long() + 6) * (1 << fraction)
    if fraction == 3:
        code = torch.where(torch.isfinite(x), code + torch.where(x < 0, 128, 0), 127)
    else:
        code = torch.where(torch.isfinite(x), torch.where(x > 0, code.clamp(min=1), code), 255)
    return code.to(torch.uint8)


def decode(code, scale, fraction):
    c = code.long()
    magnitude = c & 127 if fraction == 3 else c
    exponent, part = magnitude >> fraction, (magnitude & ((1 << fraction) - 1)).double() / (1 << fraction)
    y = torch.where(exponent > 0, 1.0 + part, part) * 2.0 ** (exponent.clamp(min=1).double() - 7.0)
    y = torch.where(each(scale, c.numel()) == 0, 0.0, y * 2.0 ** (each(scale, c.numel()).double() - 127.0))
    if fraction == 3:
        y = torch.where(magnitude == 127, math.nan, torch.where(c >= 128, -y, y))
    return y


# ---- the step ----------------------------------------------------------------------------------------------------------


def coefficient(sumsq, max_norm, grad_scale):
    norm = math.sqrt(sumsq) * abs(grad_scale)
    return grad_scale * (max_norm / norm if max_norm > 0 and norm > max_norm else 1.0)


def step64(theta, g, m, v, t, lr, beta1, beta2, eps, decay, c):
    """theta', m', v' in 64 bits, and bounds on how far fp32 arithmetic may be from them.

    Every constant and every operation is off by 2^-24 relative at most.  m': c, c g, 1 - b1, the product, the sum: 5.
    v': twice c and c g, the square, 1 - b2, the product, the sum: 8.  The step's size: m' and speed and their product 7; the
    root's half of v' and itself 5, spread, product, sum and eps 4; the division 2 ulp = 4: 20 of
    the sizes of its terms.  theta': keep, product 2, sum 1.  All rounded up by a quarter for the terms of second order and fused
    operations in another order."""
    g = g * c
    m1, v1 = beta1 * m + (1.0 - beta1) * g, beta2 * v + (1.0 - beta2) * g * g
    speed, spread = lr / (1.0 - beta1 ** t), 1.0 / math.sqrt(1.0 - beta2 ** t)
    down = torch.sqrt(v1) * spread + eps
    out = theta * (1.0 - lr * decay) - speed * m1 / down
    m_size = (beta1 * m).abs() + ((1.0 - beta1) * g).abs()
    # fp32 numbers below 2^-126 have steps of 2^-149
    tiny = 2.0 ** -148
    return out, m1, v1, 25 * ULP * speed * m_size / down + 4 * ULP * (theta.abs() + out.abs()) + tiny, \
        6.25 * ULP * m_size + tiny, 10 * ULP * v1 + tiny


def moments32(m, v, g, beta1, beta2, c):
    """m' and r' = sqrt(v') as fp32 arithmetic gives them when each operation is rounded by itself (float64 tensors of fp32
    numbers in and out; float64 holds each result exactly or with bits enough for the second rounding to be the right one)."""
    g = f32(g * f32(c))
    m = f32(f32(m * f32(beta1)) + f32(g * f32(1.0 - beta1)))
    v = f32(f32(v * f32(beta2)) + f32(f32(g * g) * f32(1.0 - beta2)))
    return m, f32(torch.sqrt(v))
