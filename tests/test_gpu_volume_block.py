"""GPU: the example block (the token operators one after the other, on the pre-decoder's activations) against the same
block in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc
from conftest import ROOT
from paper_2604_12841_amd import workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("volume_block", os.path.join(ROOT, "examples", "volume_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def block64(b, h, sites, batch, causal, weights):
    """The block in 64 bits from the quantised weights, without rounding activations to codes or bf16."""
    n, H, Hk, D = h.shape[0], b.heads, b.kv_heads, b.head_dim

    def norm(x):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    h = h.double()
    qkv = (norm(h) @ weights["qkv"].t()).view(n, H + 2 * Hk, D)
    flat = sites.expand(batch, n // batch, 4).reshape(n, 4)
    qk = tc.rope64(qkv[:, :H + Hk], flat, b.sections, 100.0, False, False)
    q, k = (x.reshape(batch, n // batch, -1, D) for x in (qk[:, :H], qk[:, H:]))
    a, _, _ = tc.attention64(q, k, qkv[:, H + Hk:].reshape(batch, n // batch, Hk, D), sites, sites, D ** -0.5, b.cap, b.slopes, causal, 0)
    h = h + norm(a.reshape(n, -1)) @ weights["out"].t()
    u = norm(h) @ weights["up"].t()
    u = u / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (u + 0.044715 * u ** 3)))
    return h + norm(u) @ weights["down"].t()


@pytest.mark.parametrize("codes,causal,d,T,batch", [("e4m3", False, 5, 5, 3), ("int8", True, 5, 7, 2), ("int8", False, 3, 1, 1)])
def test_block(example, codes, causal, d, T, batch):
    layers = workload.layer_spec(3, 128)
    pre = pdx.Predecoder(workload.he_normal_weights(layers, seed=3), d, T, layers, "bf16", max_batch=batch)
    det, _ = workload.make_inputs(d, T, batch, 0.02, 0.02, seed=4)
    sites = pdx.volume_sites(d, T)
    tokens = batch * sites.shape[0]
    h = torch.empty(tokens, 128, dtype=torch.bfloat16, device="cuda")
    pre.activations(torch.from_numpy(det.view("int64")).cuda(), 1, h)
    block = example.VolumeBlock(tokens, codes=codes)
    start = h.clone()
    left = block.run(h, sites, batch, causal=causal)
    torch.cuda.synchronize()
    got = h.double() + left.double()
    weights = {n: w[0].double() * w[1].double()[:, None] for n, w in
               (("qkv", block.w_qkv), ("out", block.w_out), ("up", block.w_up), ("down", block.w_down))}
    want = block64(block, start, sites, batch, causal, weights)
    # Each activation entering a product carries its code's rounding: E4M3 2^-4 of the value at most, 2^-5.2 rms; int8 half a step of
    # max / 127, a share of 0.29 / 127 x (max / rms <= 11) = 2.5 % rms.  Products of many independent terms keep the relative size;
    # four of them in a row add in squares, the attention's softmax of scores (rms under 3, capped) may move them by the scores' error again: 3 x 2.7 %. A tenth
    # of what the block adds bounds that.
    added = (want - start.double()).norm()
    assert (got - want).norm() <= 0.1 * added
    assert torch.isfinite(got).all()


def test_command(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["volume_block.py", "--d", "5", "--T", "5", "--batch", "2"])
    example.main()
    assert "tokens" in capsys.readouterr().out
