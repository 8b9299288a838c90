"""ams_assign_pages goes by the batch and the bound of the lengths alone: one table serves all layers and heads.  Against the plain allocator."""
import numpy as np
import pytest
import torch

import test_gpu_pages
from paper_2605_23200_amd import binding as B

pytestmark = pytest.mark.gpu


def _mixed(batch, t_max, seed):
    rng = np.random.default_rng(seed)
    had = rng.integers(0, t_max + 1, batch)
    return had, np.where(rng.random(batch) < 0.4, np.minimum(had + 1, t_max), rng.integers(0, t_max + 1, batch))


@pytest.mark.parametrize("other", [dict(n_layers=32, n_kv_heads=8), dict(n_layers=70000), dict(n_kv_heads=300, group=300), dict(head_dim=96)])
def test_sizes_that_it_does_not_use(other, monkeypatch):
    """As a model's parameters have them: more (layer, sequence, head) units than a launch over units takes, other head sizes."""
    plain = B.make_params
    monkeypatch.setattr(B, "make_params", lambda **kw: plain(**dict(kw, **other)))
    had, want = _mixed(256, 300, 1)
    test_gpu_pages._case(had, want, 300, 2000)


@pytest.mark.parametrize("batch,t_max", [(65536, 40), (70001, 33)])
def test_very_large_batches(batch, t_max):
    had, want = _mixed(batch, t_max, 2)
    test_gpu_pages._case(had, want, t_max, batch // 2)
