"""Checks of arguments in the binding of heinsen_attention that need no GPU: what they refuse never reaches a kernel."""
import pytest
import torch


@pytest.fixture(scope="module")
def ha():
    from paper_2311_06281_b200 import build_ext, heinsen_attention
    build_ext.build()
    heinsen_attention.lib()
    return heinsen_attention


def test_a_kept_workspace_is_contiguous_bytes_of_the_calls_device(ha):
    gpu, host = torch.device("cuda", 0), torch.device("cpu")
    ws = torch.empty(512, dtype=torch.uint8)
    ha._space_ok(ws, host)
    with pytest.raises(ValueError, match="workspace is on cpu"):
        ha._space_ok(ws, gpu)
    with pytest.raises(ValueError, match="workspace is on meta"):
        ha._space_ok(torch.empty(512, dtype=torch.uint8, device="meta"), gpu)
    for bad in (ws.view(torch.float32), ws[::2], torch.empty(512, dtype=torch.int8)):
        with pytest.raises(ValueError, match="contiguous uint8"):
            ha._space_ok(bad, host)
