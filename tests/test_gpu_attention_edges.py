"""decay_attention and the norms at the edges of what they accept: foreign workspaces, empty batches, states that a decay of
zero has to forget, derivatives and in-place updates as autograd sees them."""
import pytest
import torch

from attention_testlib import attention64, close, leaf64
from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_workspace_of_the_host_is_refused(ha):  # noqa: F811
    q, k, v, log_a, s0 = make(1, 40, 2, 2, 2, 2, 64, 64, BF16, state=True)
    ws = ha.workspace(q, k, v, log_a)
    for bad in (ws.cpu(), torch.empty(ws.numel(), device=DEV)):
        for grad in (False, True):
            with pytest.raises(ValueError, match="workspace"):
                ha.decay_attention(q.detach().requires_grad_(grad), k, v, log_a, s0, workspace=bad)
