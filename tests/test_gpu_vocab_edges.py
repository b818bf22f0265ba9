"""The embedding, verified drafts and distillation where a program reuses what it has: one
workspace for batches of every size, and other calls that the tests of each operator do not make."""

import numpy as np
import pytest
import torch

from gpu_util import require_gpu, to_np
from oracle import vocab

pytestmark = pytest.mark.gpu


def test_embedding_gradients_of_many_sizes_in_the_workspace_of_the_largest():
    rbp = require_gpu()
    rng = np.random.default_rng(1)
    V, d, most = 700, 512, 40000
    ws = rbp.workspace(rbp.RBP_OP_EMBED_BWD, most, d, V)
    dx = torch.from_numpy(rng.integers(-4, 5, (most, d)).astype(np.float32)).cuda()
    y = torch.from_numpy(np.where(rng.random(most) < 0.5, 3, rng.integers(0, V, most))
                         .astype(np.int32)).cuda()
    # (4096 slices of 8 positions at 32768 tokens, more than the largest batch has)
    for T in (1, 513, 4097, 8193, 12289, 32768, 32769, most):
        ws.fill_(255)
        dW = torch.full((V, d), 7.0, device="cuda")
        print(f"[workspace] embed_bwd T={T}", flush=True)
        rbp.policy_embed_bwd(dx[:T], y[:T], None, dW, ws)
        want = torch.zeros((V, d), dtype=torch.float64, device="cuda")
        want.index_add_(0, y[:T].long(), dx[:T].double())
        assert torch.equal(dW.double(), want)  # small integers: exact
