"""AdamW on a tensor of more than 2^32 elements: elements whose number passes 32 bits are stepped, and their random bits are their own."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from adamw_reference import BLOCK, codes, key, scales, step32, update
from rows_reference import close

pytestmark = pytest.mark.gpu
B1, B2 = 0.9, 0.999
LOW = 0xFFFFFFFF


def bits_from(first, n, k):
    i = torch.arange(first, first + n, device="cuda")
    x = (((i & LOW) ^ (k & LOW)) + (k >> 32) + (i >> 32) * 0x85EBCA6B) & LOW
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & LOW
    x = ((x ^ (x >> 15)) * 0x846CA68B) & LOW
    return x ^ (x >> 16)


def test_elements_beyond_32_bits():
    n = (1 << 32) + 10 * BLOCK + 77                    # 26 GB of parameters, gradients and states
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough device memory")
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, r = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(-(-n // BLOCK), device="cuda") for _ in range(2))
    gen = torch.Generator("cuda").manual_seed(6)
    at = [(0, 4 * BLOCK), ((1 << 31) - BLOCK, 2 * BLOCK), ((1 << 32) - BLOCK, 3 * BLOCK), (n - 77 - BLOCK, BLOCK + 77)]
    for b, k in at:
        p[b:b + k] = torch.randn(k, generator=gen, device="cuda").bfloat16()
        g[b:b + k] = torch.randn(k, generator=gen, device="cuda").bfloat16()
    old = [p[b:b + k].clone() for b, k in at]
    step, lr = torch.tensor([1], device="cuda"), torch.tensor([1e-2], device="cuda")
    tb.AdamW([p], [g], [m], [r], [ms], [vs]).step(step, lr, B1, B2, 1e-8, None, 12)
    for (b, k), w in zip(at, old):
        s = slice(b, b + k)
        zero = torch.zeros(k, device="cuda")
        m1, v1 = step32(zero, zero, g[s].float(), B1, B2)
        close(p[s], *update(w, m1, v1, 1, float(lr), 0.0, B1, B2, 1e-8))
        sm, sv = scales(m1.double(), v1.double())
        blocks = slice(b // BLOCK, -(-(b + k) // BLOCK))
        assert torch.equal(ms[blocks].double(), sm) and torch.equal(vs[blocks].double(), sv)
        bits = bits_from(b, k, key(12, 1, 0))
        assert torch.equal(m[s].view(torch.float8_e4m3fn).double(), torch.copysign(codes(m1.double(), sm, bits & 0xFFFF), m1.double()))
        root = torch.sqrt(v1.double()).float().double()
        assert torch.equal(r[s].view(torch.float8_e4m3fn).double(), torch.maximum(codes(root, sv, bits >> 16), torch.where(v1 > 0, 2.0 ** -9, 0.0)))
    assert int((p != 0).sum()) == sum(int((w != 0).sum()) for w in old)
