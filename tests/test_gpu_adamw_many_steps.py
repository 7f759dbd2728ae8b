"""States in 8 bits over hundreds of steps, against the same recurrence from separate operations: every code of every element, and how far the mean of v stands from that of fp32 states.

sqrt(v) is rounded up or down by chance, without bias.  Its square gains the variance: from a code c, a step goes to x, |x - c| = (1 - beta2) |g^2 - c^2| / (2 c), and rounding it to codes that are
s apart adds |x - c| (s - |x - c|) <= (1 - beta2) |g^2 - c^2| s / (2 c) to the mean of the square.  A code's step s is 1/16 to 1/8 of c.  While v grows towards g^2, as under a constant
gradient from zeros, that is at most s / (2 c) <= 1/16 of what the step adds.  Where squares of gradients go both ways around v, with a mean distance of at most g^2 + c^2 = 2 v on average, it is at most 1/8
of v.  The mean over n elements is off by less than 0.5 % besides (a spread of a code's step, 25 % in v, over the root of 65 536, five times)."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from adamw_reference import BLOCK, codes, element_bits, key, scales, step32

B1, B2 = 0.9, 0.999
N, STEPS, SEED = 1 << 16, 600, 5


class Recurrence:
    """m and the root of v as codes and scales, in fp32 values."""

    def __init__(self, device):
        self.m, self.r = (torch.zeros(N, device=device, dtype=torch.float64) for _ in range(2))      # codes
        self.ms, self.vs = (torch.zeros(N // BLOCK, device=device, dtype=torch.float64) for _ in range(2))
        self.device = device

    def values(self):
        return tuple((x * s.repeat_interleave(BLOCK)).float() for x, s in ((self.m, self.ms), (self.r, self.vs)))

    def step(self, t, g):
        m, r = self.values()
        m, v = step32(m, r * r, g, B1, B2)
        self.ms, self.vs = scales(m.double(), v.double())
        bits = element_bits(key(SEED, t, 0), N, self.device)
        self.m = torch.copysign(codes(m.double(), self.ms, bits & 0xFFFF), m.double())
        root = torch.sqrt(v.double()).float().double()                                                # rounded once: 53 bits are more than 2 x 24 + 2
        self.r = torch.maximum(codes(root, self.vs, bits >> 16), torch.where(v > 0, 2.0 ** -9, 0.0))


def gradient(kind, t, device):
    if kind == "constant":
        return torch.full((N,), 0.37, device=device)
    gen = torch.Generator(device).manual_seed(t)
    return torch.randn(N, generator=gen, device=device) * 0.37


def check_means(kind, m, r, v32):
    v = (r.double() ** 2).mean()
    assert -0.005 < float(v / v32.double().mean() - 1) < (1 / 16 if kind == "constant" else 1 / 8) + 0.005
    if kind == "constant":
        assert abs(float(m.double().mean()) / (0.37 * (1 - B1 ** STEPS)) - 1) < 0.005


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["constant", "random"])
def test_every_code_of_many_steps(kind):
    want = Recurrence("cuda")
    p = torch.zeros(N, device="cuda")
    g = torch.empty(N, device="cuda")
    m, r = (torch.zeros(N, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(N // BLOCK, device="cuda") for _ in range(2))
    adamw = tb.AdamW([p], [g], [m], [r], [ms], [vs])
    lr, step = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    v32 = torch.zeros(N, device="cuda")
    for t in range(1, STEPS + 1):
        g.copy_(gradient(kind, t, "cuda"))
        step.fill_(t)
        adamw.step(step, lr, B1, B2, 1e-8, None, SEED)
        want.step(t, g)
        v32 = step32(v32, v32, g, B1, B2)[1]
        if t % 50 == 0 or t < 5:
            assert torch.equal(m.double(), want.m) and torch.equal(r.double(), want.r)
            assert torch.equal(ms.double(), want.ms) and torch.equal(vs.double(), want.vs)
    check_means(kind, *want.values(), v32)


@pytest.mark.parametrize("kind", ["constant", "random"])
def test_means_of_the_recurrence(kind):
    """The recurrence by itself, without a GPU: the bound holds for what is asked of the kernel."""
    want, v32 = Recurrence("cpu"), torch.zeros(N)
    for t in range(1, STEPS + 1):
        g = gradient(kind, t, "cpu")
        want.step(t, g)
        v32 = step32(v32, v32, g, B1, B2)[1]
        if t % 300 == 0:
            m, r = want.values()
            print(t, float((r.double() ** 2).mean() / v32.double().mean() - 1))
    check_means(kind, *want.values(), v32)
