"""The operators together, as examples/decode_step.py runs them: each stage against its own definition on the
stage before, the sampled tokens among those the constraints leave, and the whole chain in a graph.

The 8-bit stage is exact given its inputs (integers, one scale a row): its tolerance is that of test_gpu_norm.py.
The head's is that of test_gpu_matmul_w4.py for 8-bit rows."""
from __future__ import annotations

import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _fill(tail, seed):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)
    tail.hidden.copy_(torch.randn(tail.hidden.shape, generator=g, device="cuda"))
    tail.residual.copy_(torch.randn(tail.residual.shape, generator=g, device="cuda") * 2)


@pytest.mark.parametrize("batch,V,D", [(1, 5000, 512), (7, 20011, 1024), (40, 9001, 640)])
def test_each_stage(example, batch, V, D):
    import torch

    import paper_2606_01927_amd as alb

    tail = example.build(batch, V, D)
    _fill(tail, 3)
    h = tail.hidden.double().cpu().numpy() + tail.residual.double().cpu().numpy()
    tail.norm()
    tail.head()
    raw = tail.logits.clone()
    tail.adjust()
    adjusted = tail.logits.clone()
    w = tail.norm._keep[1].double().cpu().numpy()
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5) * w
    q, scale = tail.norm.result.q.cpu().numpy().astype(np.float64), tail.norm.result.scale.double().cpu().numpy()
    assert np.abs(q - y / (np.abs(y).max(1, keepdims=True) / 127)).max() <= 0.5 + 127 * 3e-5
    head = tail.head._keep[2]
    packed = head.q.cpu().numpy()
    dense = np.empty((V, D))
    dense[:, 0::2], dense[:, 1::2] = packed & 15, packed >> 4
    dense = (dense - 8) * np.repeat(head.scales.double().cpu().numpy(), 128, 1)
    x = q * scale[:, None]
    tol = 4 * np.sqrt(D) * 2.0 ** -24 * (np.abs(x) @ np.abs(dense).T)
    assert (np.abs(raw.double().cpu().numpy() - x @ dense.T) <= tol).all()
    c = tail.adjust._keep[2]
    idx = c.mask_index.cpu().numpy()
    words = c.mask.cpu().numpy().view(np.uint32)
    bits = ((words[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(words.shape[0], -1)[:, :V] != 0
    want = raw.cpu().numpy()
    ids = c.bias_ids.cpu().numpy().reshape(batch, -1)
    for b in range(batch):
        want[b, ids[b]] = -np.inf
        if idx[b] >= 0:
            want[b, ~bits[idx[b]]] = -np.inf
    assert np.array_equal(adjusted.cpu().numpy(), want)
    # the tokens are ones that the biases and masks leave
    ids2, lps2, _, _, _ = alb.sample_step(adjusted, tail.seed, 0, params=tail.params)
    tail.hidden.zero_()
    assert (tail.logits == adjusted).all() and torch.isfinite(lps2).all() and (ids2 >= 0).all()
    for b in range(batch):
        assert np.isfinite(want[b, int(ids2[b])])


def test_steps_and_tokens(example):
    import torch

    tail = example.build(9, 6000, 512)
    seen = []
    for i in range(4):
        _fill(tail, i)
        ids, lps, flags = tail.step()
        assert torch.equal(ids, tail.next_tokens) and (ids >= 0).all() and torch.isfinite(lps).all() and (flags == 0).all()
        for b in range(9):
            assert torch.isfinite(tail.logits[b, int(ids[b])])
        seen.append(ids.clone())
    n = tail.state.len.cpu().numpy()
    got = [set(tail.state.ids[b, :n[b]].cpu().numpy()[(tail.state.counts[b, :n[b]].cpu().numpy() & 0x7fffffff) > 0]) for b in range(9)]
    for b in range(9):
        assert got[b] == {int(s[b]) for s in seen}


def test_chain_in_a_graph(example):
    import torch

    tail = example.build(6, 8000, 1024)
    _fill(tail, 1)
    keep = tail.residual.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tail.norm(), tail.head(), tail.adjust()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            tail.norm(), tail.head(), tail.adjust()
    torch.cuda.synchronize()
    for seed in range(4):  # replays, each with eager work and a synchronisation in between
        _fill(tail, seed)
        keep.copy_(tail.residual)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got, res = tail.logits.clone(), tail.residual.clone()
        tail.residual.copy_(keep)
        tail.norm(), tail.head(), tail.adjust()
        torch.cuda.synchronize()
        assert torch.equal(got, tail.logits) and torch.equal(res, tail.residual)
