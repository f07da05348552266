"""The status word of a cache attention workspace."""
import pytest
import torch

from tests.test_gpu_cache import sb  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_status_of_what_is_no_workspace_here(sb):  # noqa: F811
    """A workspace of another device is not ordered behind this one's stream, and host memory has no status."""
    ws = sb.make_cache_workspace(1, 1, 1, 64)
    assert sb.sol_attn_cache_read_status(ws) == sb.SOL_OK
    for bad in (torch.zeros(4096, dtype=torch.uint8), ws[:100], ws.float()):
        with pytest.raises(ValueError):
            sb.sol_attn_cache_read_status(bad)
