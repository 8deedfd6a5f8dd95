"""Modules of the whole models (arxiv 2411.01238, Section 4.2) are called as modules whatever their operators run in: hooks on them run."""
import pytest
import torch

from paper_2411_01238_amd import model_step as ms
from paper_2411_01238_amd import sdrop

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["vit", "gpt"])
def test_every_module_is_called(name):
    cfg = {"vit": dict(image=16, patch=2, d=128, n_layers=2, n_head=2), "gpt": dict(context=32, d=128, n_layers=2, n_head=2)}[name]
    shape = {k: v for k, v in cfg.items() if k in ("image", "context")}
    batch = ms.synthetic_batch(name, seed=1, dtype=torch.float16, batch=8, **shape)
    called = {}
    for ops in ms.OPS:
        model = ms.MODELS[name]("dense", 0.0, dtype=torch.float16, ops=ops, resid_p=0.1, **cfg).train()
        seen = called[ops] = []
        for n, m in model.named_modules():
            if n and not isinstance(m, torch.nn.ModuleList):
                m.register_forward_hook(lambda mod, args, out, n=n: seen.append(n))
        model.loss(batch).backward()
        assert set(seen) == {n for n, m in model.named_modules() if n and not isinstance(m, torch.nn.ModuleList)}, ops
    # and as often
    assert sorted(called["torch"]) == sorted(called["sdrop"])
    assert sdrop.status() == 0
