"""What the paged cache's calls flag and what they do not."""
import pytest
import torch

import test_gpu_kv_cache as C

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def test_sequences_without_rows_may_hold_more_than_the_call_has_pages_for(S):
    both = C.Both(S, 3, 3, 2, 64, 32)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = torch.randn((80, 2, 2, 64), device=DEV)
    both.append(x[:, 0], x[:, 1], [75, 3, 2], status=status)
    both.table = both.table[:, :1].contiguous()                       # a page a sequence: the first one's others are not needed
    both.append(x[:9, 0], x[:9, 1], [0, 4, 5], status=status)
    both.check()
    assert status.item() == 0
    S.kv_read(both.cache, both.table, C._i32(both.held), C._i32([0, 0, 0, 0]), 1, torch.float32, status)
    torch.cuda.synchronize()
    assert status.item() == 0
