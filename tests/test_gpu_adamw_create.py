"""An AdamW list that is stepped as soon as it is made, on a stream that does not wait for any other."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from adamw_reference import step32, update
from rows_reference import close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count,n", [(1, 100_000_000), (20_000, 1000)])
def test_first_step_on_a_stream_of_its_own(count, n):
    """Lists whose tables take a megabyte and more: of tiles, of tensors."""
    total = count * n
    p, g = torch.randn(total, device="cuda"), torch.randn(total, device="cuda")
    m, v = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
    old, m1, v1 = p.clone(), *step32(m, v, g, 0.9, 0.999)
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-2, device="cuda")
    stream = torch.cuda.Stream()
    lists = [list(x.split(n)) for x in (p, g, m, v)]
    torch.cuda.synchronize()
    adamw = tb.AdamW(*lists)
    adamw.step(step, lr, stream=stream)
    stream.synchronize()
    assert torch.equal(m, m1) and torch.equal(v, v1)
    for b in range(0, total, 10_000_000):
        part = slice(b, b + 10_000_000)
        close(p[part], *update(old[part], m1[part], v1[part], 1, float(lr), 0.0, 0.9, 0.999, 1e-8))
