"""Whole models (arxiv 2411.01238, Section 4.2) whose norms, residual adds, attention and element dropout run in the library's
kernels: against the same model of torch operations in float64 on the CPU, with the float64 definitions' masks.  The 16-bit model
rounds every activation: the tolerance is that of the other whole-model test, a chain of fp16 roundings."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import sdrop_oracle as orc
from oracle import transformer_oracle as torc
from paper_2411_01238_amd import model_step as ms
from paper_2411_01238_amd import sdrop
from _util import errors, kernel_names

pytestmark = pytest.mark.gpu

SMALL = {
    "mlp": dict(in_dim=256, hidden=512, n_hidden=1, n_out=10),
    "vit": dict(image=16, patch=2, d=384, n_layers=2, n_head=3, n_out=10),
    "gpt": dict(vocab=65, context=64, d=384, n_layers=2, n_head=6),
}
BATCH = {"mlp": 384, "vit": 8, "gpt": 8}


def _element_dropout(masks):
    """F.dropout with the masks of the definitions, asked for in the order in which the model's layers call."""
    def dropout(x, p, training=True):
        seed, call = next(masks)
        m = x.reshape(-1, x.shape[-1])
        keep = torch.from_numpy(torc.element_keep(*m.shape, p, seed, call)).view(x.shape)
        return torch.where(keep, x * torc.element_scale(p), torch.zeros_like(x))
    return dropout


@pytest.mark.parametrize("name", ["mlp", "vit", "gpt"])
@pytest.mark.parametrize("kind", ["dense", "dropout_dense", "sparsedrop"])
def test_model_of_the_librarys_operators_matches_float64(name, kind, monkeypatch):
    print("model", name, kind, flush=True)
    torch.manual_seed(3)
    cfg = SMALL[name]
    extra = {} if name == "mlp" else dict(resid_p=0.2)
    p = 0.0 if kind == "dense" else 0.4
    model = ms.MODELS[name](kind, p, dtype=torch.float16, ops="sdrop", **cfg, **extra).train()
    ref = ms.MODELS[name]("block_dropout_dense" if kind == "sparsedrop" else kind, p, dtype=torch.float64, device="cpu",
                          keep_fn=lambda MB, KB, p_, seed, call: np.asarray(orc.mask(MB, KB, p_, seed, call)), **cfg, **extra).train()
    ref.load_state_dict({k: v.detach().cpu().double() for k, v in model.state_dict().items()})
    shape = {k: v for k, v in cfg.items() if k in ("in_dim", "n_out", "image", "context", "vocab")}
    for step in range(2):
        # the order of the element dropouts: of each layer's input where it has one, of what is added to the residual stream
        order = []
        each = kind == "dropout_dense"
        if name == "mlp":
            order = [(i, step) for i in range(3)] if each else []
        else:
            for b in range(cfg["n_layers"]):
                order += [(10 * b, step), (10 * b + 1, step)] if each else []
                order += [(10 * b + 4, step)]
                order += [(10 * b + 2, step), (10 * b + 3, step)] if each else []
                order += [(10 * b + 5, step)]
            if name == "gpt" and each:
                order += [(10 * cfg["n_layers"], step)]
        batch = ms.synthetic_batch(name, seed=step, dtype=torch.float16, batch=BATCH[name], **shape)
        rbatch = tuple(t.cpu().double() if t.is_floating_point() else t.cpu() for t in batch)
        for mdl in (model, ref):
            for prm in mdl.parameters():
                prm.grad = None
        loss = model.loss(batch)
        loss.backward()
        masks = iter(order)
        with monkeypatch.context() as m:
            m.setattr(F, "dropout", _element_dropout(masks))
            rloss = ref.loss(rbatch)
        assert next(masks, None) is None
        rloss.backward()
        torch.cuda.synchronize()
        assert abs(loss.item() - rloss.item()) <= 2e-2 * abs(rloss.item()), (step, loss.item(), rloss.item())
        for (n, prm), (_, rprm) in zip(model.named_parameters(), ref.named_parameters()):
            got, want = prm.grad.double().cpu().numpy(), rprm.grad.numpy()
            assert np.all(np.isfinite(got)), n
            fro, _ = errors(got, want)
            assert fro <= 3e-2, "step %d, %s: relative Frobenius error %.3e" % (step, n, fro)
    assert sdrop.status() == 0


def test_the_librarys_kernels_run_and_evaluation_drops_nothing():
    cfg = SMALL["gpt"]
    a = ms.GPT("dropout_dense", 0.5, dtype=torch.float16, ops="sdrop", resid_p=0.5, **cfg)
    batch = ms.synthetic_batch("gpt", seed=1, batch=8, **{k: cfg[k] for k in ("context", "vocab")})
    a.train()
    with torch.no_grad():
        names = " ".join(kernel_names(lambda: a(batch[0])))
    for k in ("attn_fwd_kernel", "norm_fwd_kernel", "dropout_kernel"):
        assert k in names, k
    b = ms.GPT("dense", 0.0, dtype=torch.float16, **cfg).eval()
    b.load_state_dict(a.state_dict())
    a.eval()
    with torch.no_grad():
        x, y = a(batch[0]).double().cpu().numpy(), b(batch[0]).double().cpu().numpy()
    # two fp16 chains of the same model, each about 20 roundings long
    assert errors(x, y)[0] <= 20 * 2.0 ** -10
    # a block called by itself
    h = a.blocks[0](a.tok(batch[0]) + a.pos[:64])
    assert errors(h.double().detach().cpu().numpy(), b.blocks[0](b.tok(batch[0]) + b.pos[:64]).double().detach().cpu().numpy())[0] <= 20 * 2.0 ** -10
