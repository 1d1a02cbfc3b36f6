"""AdamW over many tensors: outputs of the moments' values that lie next to each other, in any order."""

import pytest
import torch

from tests.test_gpu_adamw_multi import Set

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_state_values_side_by_side(dt):
    from paper_2309_01226_amd import ops
    sizes = [257, 0, 1, 1000, 4096]
    s = Set(sizes, 8, "fp32")
    apart = [[torch.zeros(n, device="cuda", dtype=dt) for n in sizes] for _ in range(2)]
    ops.adamw_multi_state(s.table, *apart)
    whole = torch.zeros(2 * sum(sizes), device="cuda", dtype=dt)
    cuts = list(whole.split(sizes[::-1] + sizes[::-1]))[::-1]  # from the end on, nothing between them
    ops.adamw_multi_state(s.table, cuts[:len(sizes)], cuts[len(sizes):])
    torch.cuda.synchronize()
    for a, b in zip(apart[0] + apart[1], cuts):
        assert torch.equal(a, b)
    with pytest.raises(RuntimeError):
        ops.adamw_multi_state(s.table, apart[0], apart[0])
