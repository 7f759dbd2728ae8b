"""States in 8 bits, bit for bit: every code is that of m and of the correctly rounded root of v, both from separately rounded fp32 operations, rounded up by the element's random bits."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from adamw_reference import BLOCK, codes, element_bits, key, scales, step32

pytestmark = pytest.mark.gpu
F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
B1, B2 = 0.9, 0.999


def root_of(v):
    """Rounded once: a root in 53 bits that is rounded to 24 is the root rounded to 24 (53 >= 2 x 24 + 2)."""
    return torch.sqrt(v.double()).float().double()


def check(n, pt, gt, master, scale, shift, eps, t, seed=7, factor=1.0, zeros=False):
    g = torch.Generator("cuda").manual_seed(n + t)
    normal = lambda: torch.randn(n + shift, generator=g, device="cuda")[shift:]                      # noqa: E731
    nb = -(-n // BLOCK)
    grad = (normal() * torch.exp(factor * normal()) * scale).to(gt)
    if zeros:
        grad[torch.rand(n, generator=g, device="cuda") < 0.5] = 0
    p = normal().to(pt)
    w = normal() if master else None
    m, r = ((torch.randint(0, 0x78, (n + shift,), generator=g, device="cuda").to(torch.uint8)[shift:]) for _ in range(2))
    if zeros:
        r[grad == 0] = 0
    ms, vs = ((2.0 ** torch.randint(-9, -6, (nb,), generator=g, device="cuda")).float() * 2.0 ** round(torch.log2(torch.tensor(scale)).item()) for _ in range(2))
    mv, rv = (x.view(E4M3).float() * s.repeat_interleave(BLOCK)[:n] for x, s in ((m, ms), (r, vs)))
    m2, v2 = step32(mv, rv * rv, grad.float(), B1, B2)
    sm, sv = scales(m2.double(), v2.double())
    step, lr = torch.tensor([t], device="cuda"), torch.tensor([1e-3], device="cuda")
    tb.AdamW([p], [grad], [m], [r], [ms], [vs], [w] if master else None).step(step, lr, B1, B2, eps, None, seed)
    assert torch.equal(ms.double(), sm[:nb]) and torch.equal(vs.double(), sv[:nb])
    bits = element_bits(key(seed, t, 0), n, "cuda")
    assert torch.equal(m.view(E4M3).double(), torch.copysign(codes(m2.double(), sm, bits & 0xFFFF), m2.double()))
    want = torch.maximum(codes(root_of(v2), sv, bits >> 16), torch.where(v2 > 0, 2.0 ** -9, 0.0))
    off = r.view(E4M3).double() != want
    assert not off.any(), "%d of %d codes of the root are another" % (int(off.sum()), n)


@pytest.mark.parametrize("pt,gt,master", [(F32, F32, False), (BF16, BF16, False), (BF16, F32, True), (F16, F16, False)])
def test_codes_of_many_elements(pt, gt, master):
    """Enough of them for a root one unit off in its last place to show: one in a million elements stands that near to a border between two codes."""
    check(20_000_000, pt, gt, master, 1e-3, 0, 1e-8, 9)
    check(20_000_000, pt, gt, master, 1e-2, 0, 1e-8, 100, zeros=True)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("scale,eps", [(1.0, 1e-8), (1e8, 1e-8), (1e-12, 1e-8), (1e-12, 1e-16), (1e-18, 1e-25)])
def test_codes_of_every_size(scale, eps, shift):
    """Roots whose squares are near the ends of the range, by vectors and by element, wide blocks; eps beside which small roots count."""
    for n in (1, 255, 300, 4_000_001):
        check(n, F32, F32, False, scale, shift, eps, 3, factor=2.0)
