"""The operators around the aggregation used together: the expert layer of examples/ against the same
layer in plain torch, float32 with autograd, on the CPU, with the experts that the layer chose."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import layer_refs as ref
import paper_2507_16991_amd as mp

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("expert_layer",
                                                  os.path.join(ROOT, "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(layer, ptr, x, idx, keep, scale, We=None):
    """The layer in float32; leaves is what gradients are taken of."""
    leaves = dict(x=x, gamma=layer.gamma, beta=layer.beta, Wr=layer.Wr, We=layer.We if We is None else We)
    leaves = {n: t.detach().float().cpu().requires_grad_(True) for n, t in leaves.items()}
    N, F = x.shape
    w, parts = F // layer.groups, []
    for a, b in zip(ptr[:-1], ptr[1:]):
        if a < b:
            v = leaves["x"][a:b].view(b - a, layer.groups, w)
            m = v.mean((0, 2), keepdim=True)
            parts.append(((v - m) / ((v - m).square().mean((0, 2), keepdim=True) + 1e-5).sqrt()).view(b - a, F))
    h = torch.nn.functional.silu(torch.cat(parts) * leaves["gamma"] + leaves["beta"])
    logits = h @ leaves["Wr"][0]
    weight = torch.softmax(logits.gather(1, idx), 1)
    y = torch.stack([(h[:, None] @ leaves["We"][idx[:, j]])[:, 0] * weight[:, j:j + 1]
                     for j in range(layer.k)]).sum(0)
    share = torch.bincount(idx.view(-1), minlength=layer.E).float() / idx.numel()
    balance = layer.E * (share * torch.softmax(logits, 1).mean(0)).sum()
    z = torch.logsumexp(logits, 1).square().mean()
    return leaves["x"] + y * keep * scale, torch.stack([balance, z]), leaves


def far(a, b):
    a, b = ref.f64(a), ref.f64(b)
    return np.linalg.norm(a - b) / np.linalg.norm(b)


@pytest.mark.parametrize("act_p", [0.0, 0.25])
def test_training_step(act_p):
    ex = example()
    layer = ex.ExpertLayer(F=64, E=8, k=2, groups=8, p=act_p, seed=3)
    ptr, x = ex.batch(700, 23, 64, seed=1)
    out, losses, saved = layer.forward(ptr, x, 7)
    dout = torch.randn(700, 64, generator=torch.Generator().manual_seed(2)).bfloat16().to(x.device)
    dloss = torch.tensor([3.0, 0.5], device=x.device)
    grads = layer.backward(saved, dout, dloss)

    limit = round(65536 * act_p)
    _, keep = ref.dropout(np.ones((700, 64)), act_p, 3, t=7)
    idx = saved["idx"].long().cpu()
    want, losses_r, leaves = plain(layer, ptr.tolist(), x, idx, torch.from_numpy(keep.copy()).float(),
                                   65536 / (65536 - limit))
    (want * dout.float().cpu()).sum().add((losses_r * dloss.cpu()).sum()).backward()
    # bf16 holds h, the experts' inputs and the gradients between the products: 2^-9 of each in the norm,
    # about ten of them in a row
    assert far(out, want) < 0.02
    assert far(losses, losses_r) < 0.01
    for name, g in grads.items():
        assert far(g, leaves[name].grad) < 0.04, name


def test_serving_in_four_bits():
    """Equal to the plain layer with the weights' and inputs' 4-bit values."""
    ex = example()
    layer = ex.ExpertLayer(F=64, E=8, k=2, groups=8, p=0.0, seed=4)
    ptr, x = ex.batch(300, 9, 64, seed=5)
    got = layer.serve(ptr, x)
    h, _, _ = mp.group_norm(ptr, x, 8, weight=layer.gamma, bias=layer.beta, act="silu")
    idx, weight, _, _ = mp.route(mp.segment_matmul([0, 300], h, layer.Wr), 2)
    hq = ref.mx_quantize(ref.f64(h))[2]
    wq = ref.mx_quantize(ref.f64(layer.We.transpose(1, 2)).reshape(-1, 64))[2].reshape(8, 64, 64)
    i = idx.cpu().numpy()
    y = sum(ref.f64(weight)[:, j:j + 1] * np.einsum("nk,nok->no", hq, wq[i[:, j]]) for j in range(2))
    want = ref.f64(x) + y
    assert np.linalg.norm(ref.f64(got) - want) / np.linalg.norm(want) < 2.0 ** -7


def test_loss_goes_down():
    ex = example()
    layer = ex.ExpertLayer(F=64, E=8, k=2, groups=8, p=0.0, seed=6)
    ptr, x = ex.batch(2000, 50, 64, seed=7)
    target = torch.randn(2000, 64, generator=torch.Generator().manual_seed(8)).to(x.device)
    dloss = torch.zeros(2, device=x.device)
    seen = []
    for step in range(6):
        out, _, saved = layer.forward(ptr, x, step)
        diff = out.float() - target
        seen.append(float(diff.square().mean()))
        grads = layer.backward(saved, (2 * diff / diff.numel()).bfloat16(), dloss)
        layer.We = (layer.We.float() - 100.0 * grads["We"]).bfloat16()
    assert all(b < a for a, b in zip(seen, seen[1:]))
