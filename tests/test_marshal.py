"""The binding's C++ part, on the GPU: what it refuses."""
import pytest
import torch

from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from test_parity_attn_q8 import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def test_a_workspace_that_is_not_as_large_as_its_elements():
    """One byte seen as many, and every other byte of a buffer."""
    case = Case([2], [5], 2, 1, 64)
    g = case.dev()
    size = B.adt_tree_attn_q8_workspace_size(**case.shape())
    for ws in (torch.zeros(1, dtype=torch.uint8, device="cuda").expand(size), torch.zeros(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            case.call(g, ws=ws)
    case.call(g)
    case.check(g)
