"""AdamW in 64 bits, and its states in 8 bits: codes and scales as their definition says, with the random bits of each element."""
import torch

U32 = 2.0 ** -24
BLOCK = 256
LOW = 0xFFFFFFFF
M64 = (1 << 64) - 1


def mix(z):
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def key(seed, step, tensor):
    h = 0x243F6A8885A308D3
    for x in (seed, step, tensor):
        h = mix(h ^ (0x9E3779B97F4A7C15 * (x + 1) & M64))
    return h


def element_bits(k, n, device, first=0):
    i = torch.arange(first, first + n, device=device)
    x = (((i & LOW) ^ (k & LOW)) + (k >> 32) + (i >> 32) * 0x85EBCA6B) & LOW
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & LOW
    x = ((x ^ (x >> 15)) * 0x846CA68B) & LOW
    return x ^ (x >> 16)


def power(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def exponent(x):
    """Whole part of the logarithm of positive fp32 values (held as fp64)."""
    return torch.frexp(x)[1] - 1


def blocks_of(x):
    n = len(x)
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)


def scales(m, v):
    """Powers of two of each block, from the values that are numbers; m, v: fp32 values held in 64 bits."""
    def most(x):
        return blocks_of(torch.where(torch.isfinite(x), x.abs(), 0.0)).amax(1)

    return power(exponent(most(m).clamp(min=2.0 ** -119)) - 7), power((exponent(most(v).clamp(min=2.0 ** -126)) >> 1) - 7)


def codes(x, scale, bits, off=0.0):
    """Values (fp64) as multiples of their step, rounded by the 16 bits; off: x's relative error, taken upwards or downwards."""
    q = x.abs() * (1 + off) / scale.repeat_interleave(BLOCK)[:len(x)]
    unit = power(exponent(q.clamp(min=2.0 ** -100)).clamp(min=-6) - 3)
    return torch.floor((torch.floor(q / unit * 65536) + bits) / 65536) * unit


def step32(m, v, g, beta1, beta2):
    """m and v in separately rounded fp32 operations, as they are defined."""
    f = lambda x: torch.tensor(x, dtype=torch.float32, device=m.device)  # noqa: E731
    return f(beta1) * m + f(1 - beta1) * g, f(beta2) * v + f(1 - beta2) * g * g


def update(p, m, v, t, lr, decay, beta1, beta2, eps):
    """(new parameters in 64 bits, a bound of what fp32 may be off).  The update is a quotient of rounded factors (12 u: two correction factors of 4 ulp each, the
    hardware's root and division of 2 ulp); the parameter takes a product and two sums."""
    p, m, v = p.double(), m.double(), v.double()
    up = lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
    new = p - lr * decay * p - up
    return new, up.abs() * 24 * U32 + 4 * U32 * p.abs()
