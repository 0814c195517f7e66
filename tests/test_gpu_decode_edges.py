"""The operators for few sequences where they meet what they must leave alone: rows of another batch size, sequences
without rows, values that no row sees, weights of experts that a token did not choose."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_21712_amd as moe
from gpu_util import log
from test_gpu_few import inputs
from test_gpu_kv8 import HostCache, angles, attention64, filled, i32, rotate

pytestmark = pytest.mark.gpu


@pytest.fixture
def budget():
    yield moe.set_cu_budget
    moe.set_cu_budget(0)


# ---------------------------------------------------------------- graphs of one layer
def test_graphs_of_several_sizes():
    """Two batch sizes captured from one layer, and eager runs of a third between the replays: each replay returns
    the rows of its own size."""
    log("[gpu] few: graphs of several sizes")
    H, E, k, F = 256, 16, 4, 128
    x, logits, shapes, r = inputs(12, H, E, k, F, 0, 5)
    w = [(torch.randn(s, generator=r) * s[2] ** -0.5).to(torch.bfloat16).cuda() for s in shapes]
    layer = moe.MoELayerFew(12, H, E, k, F)
    x, logits = x.cuda(), logits.cuda()
    sizes = (3, 12)
    xs, ls = [x[:n].clone() for n in sizes], [logits[:n].clone() for n in sizes]
    graphs = [moe.LayerGraph(layer, a, b, *w) for a, b in zip(xs, ls)]
    for i in range(6):
        g = i % 2
        xs[g].copy_(torch.randn(xs[g].shape, generator=r).to(torch.bfloat16))
        ls[g].copy_(torch.randn(ls[g].shape, generator=r))
        want = layer.run(xs[g], ls[g], *w).clone()
        ids, wts = layer.topk_ids.clone(), layer.topk_weights.clone()
        layer.run(x[:7 + i % 3], logits[:7 + i % 3], *w)
        torch.cuda.synchronize()
        y = graphs[g].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        assert torch.equal(graphs[g].topk_ids, ids) and torch.equal(graphs[g].topk_weights, wts), i
