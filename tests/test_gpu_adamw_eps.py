"""AdamW with the smallest eps that there are, subnormal ones too: an element with no gradient and no state keeps its place, and the others divide by what the formula says."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from adamw_reference import BLOCK, step32, update
from rows_reference import close

pytestmark = pytest.mark.gpu
B1, B2, E4M3 = 0.9, 0.999, torch.float8_e4m3fn


@pytest.mark.parametrize("eps", [1.5e-45, 1e-40, 1.1754942e-38, 1.1754944e-38, 1e-37, 1e-25])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("pt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
def test_elements_with_nothing_to_do(eps, eight, pt, shift):
    n = 5000
    eps = float(torch.tensor(eps))                     # as fp32
    g = torch.Generator("cuda").manual_seed(2)
    p = torch.randn(n + shift, generator=g, device="cuda").to(pt)[shift:]
    grad = torch.randn(n + shift, generator=g, device="cuda")[shift:] * 1e-3
    grad[1000:3000] = 0                                # rows that no id named
    m, v = (torch.zeros(n + shift, dtype=E4M3 if eight else torch.float32, device="cuda")[shift:] for _ in range(2))
    scales = [[torch.zeros(-(-n // BLOCK), device="cuda")] if eight else None for _ in range(2)]
    if not eight:                                      # a state without a square: lr m / eps, where that is a number
        m[2000:2500] = eps * torch.rand(500, generator=g, device="cuda") if eps >= 1e-37 else 2e-38 if eps > 1e-41 else 0.0
    m0, v0, p0 = m.clone().float(), v.clone().float(), p.clone()
    step, lr = torch.tensor([3], device="cuda"), torch.tensor([1e-3], device="cuda")
    tb.AdamW([p], [grad], [m], [v], *scales, weight_decay=0.25).step(step, lr, B1, B2, eps)
    m1, v1 = step32(m0, v0, grad, B1, B2)
    new, err = update(p0, m1, v1, 3, float(lr), 0.25, B1, B2, eps)
    close(p, new, err)
    still = (m1 == 0) & (v1 == 0)
    assert int(still.sum()) >= 1500
    keep = (p0.float() * float(1 - 0.25 * lr)).to(pt)  # the decay alone
    close(p[still], keep[still].double(), 4 * 2.0 ** -24 * keep[still].double().abs())
