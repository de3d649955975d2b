"""The end of a decode step, from the last hidden states to the next iteration's tokens, with synthetic inputs:

    residual addition and norm to 8 bits -> 4-bit language-model head -> biases and grammar masks in place ->
    sampling with penalties, device uniforms and backfill -> penalty state

Every operator is prepared once on buffers that stay in place, as a decode loop keeps them.  A request's bias and
its grammar's mask are written into the same buffers from step to step.

    python examples/decode_step.py --batch 64 --vocab 128256 --width 4096 --steps 20
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2606_01927_amd as alb  # noqa: E402


class DecodeTail:
    """The buffers and prepared calls of one batch.  ``hidden`` [B, D] and ``residual`` [B, D] (bfloat16) are what
    the last layer leaves; step() fills ``next_tokens`` [B] from them."""

    def __init__(self, head: alb.W4Weight, norm_weight, batch: int, params: alb.SamplingParams,
                 constraints: alb.Constraints, seed: int, prompt=None, device="cuda"):
        self.V, D = head.N, head.K
        self.hidden = torch.zeros((batch, D), dtype=torch.bfloat16, device=device)
        self.residual = torch.zeros((batch, D), dtype=torch.bfloat16, device=device)
        self.norm = alb.PreparedNorm(
            self.hidden, norm_weight, eps=1e-5, residual=self.residual, normed=False, quant=True,
            out=alb.NormOut(residual=self.residual, q=torch.empty((batch, D), dtype=torch.int8, device=device),
                            scale=torch.empty(batch, dtype=torch.float32, device=device)))
        q = self.norm.result
        self.head = alb.PreparedMatmulW4(q.q, head, x_scale=q.scale)
        self.logits = self.head.result
        self.adjust = alb.PreparedAdjust(self.logits, None, constraints, out=self.logits)
        self.params, self.seed, self.steps = params, seed, 0
        self.state = alb.PenaltyState(batch, 4096, device)
        offsets, ids = prompt if prompt is not None else (None, None)
        self.state.init(self.V, prompt_offsets=offsets, prompt_ids=ids)
        self.params.state = self.state
        self.next_tokens = torch.full((batch,), -1, dtype=torch.int32, device=device)
        self.slots = torch.arange(batch, dtype=torch.int32, device=device)

    def step(self):
        """Enqueue one step; returns (ids, logprobs, flags) of the batch."""
        self.norm()
        self.head()
        self.adjust()
        ids, logprobs, _, _, flags = alb.sample_step(self.logits, self.seed, self.steps, params=self.params,
                                                     next_tokens=self.next_tokens, backfill_dest=self.slots)
        self.state.append(ids, self.V)
        self.steps += 1
        return ids, logprobs, flags


def synthetic_head(V: int, D: int, group: int, gen, device="cuda") -> alb.W4Weight:
    packed = torch.randint(0, 256, (V, D // 2), generator=gen, dtype=torch.uint8, device=device)
    scales = (0.5 + torch.rand((V, D // group), generator=gen, device=device)) * (4.0 / 4.6 / D ** 0.5)
    return alb.W4Weight(packed, scales.bfloat16())


def build(batch: int, V: int, D: int, group: int = 128, seed: int = 1, device="cuda") -> DecodeTail:
    g = torch.Generator(device=device).manual_seed(seed)
    params = alb.SamplingParams(
        temperature=torch.full((batch,), 0.8, device=device), top_k=torch.full((batch,), 40, dtype=torch.int32, device=device),
        top_p=torch.full((batch,), 0.95, device=device), repetition_penalty=torch.full((batch,), 1.1, device=device),
        frequency_penalty=torch.full((batch,), 0.2, device=device))
    # every third request follows a grammar (two states shared between them), every request bans a few tokens
    words = (V + 31) // 32
    mask = torch.randint(-2**31, 2**31 - 1, (2, words), generator=g, dtype=torch.int32, device=device)
    index = torch.arange(batch, dtype=torch.int32, device=device) % 6
    index = torch.where(index % 3 == 0, index // 3, torch.full_like(index, -1))
    bias_ids = torch.randint(0, V, (batch * 8,), generator=g, device=device).to(torch.int32)
    constraints = alb.Constraints(
        bias_offsets=torch.arange(batch + 1, dtype=torch.int64, device=device) * 8, bias_ids=bias_ids,
        bias_values=torch.full((batch * 8,), -float("inf"), device=device), mask=mask, mask_index=index.to(torch.int32))
    prompt_ids = torch.randint(0, V, (batch * 64,), generator=g, device=device).to(torch.int32)
    prompt = (torch.arange(batch + 1, dtype=torch.int64, device=device) * 64, prompt_ids)
    weight = 0.5 + torch.rand(D, generator=g, device=device)
    return DecodeTail(synthetic_head(V, D, group, g, device), weight, batch, params, constraints, seed, prompt, device)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=128256)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    tail = build(a.batch, a.vocab, a.width)
    g = torch.Generator(device="cuda").manual_seed(2)
    layer = [torch.randn((a.batch, a.width), generator=g, device="cuda").bfloat16() for _ in range(4)]

    def run(n):
        for i in range(n):  # what the layers of a model would leave
            tail.hidden.copy_(layer[i % 4])
            tail.residual.copy_(layer[(i + 1) % 4])
            out = tail.step()
        return out

    run(3)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    ids, logprobs, flags = run(a.steps)
    end.record()
    end.synchronize()
    us = begin.elapsed_time(end) / a.steps * 1e3
    print("%d x %d, width %d: %.1f us a step, %.0f tokens/s" % (a.batch, a.vocab, a.width, us, a.batch / us * 1e6))
    print("tokens", ids[:8].tolist(), "logprobs", [round(v, 3) for v in logprobs[:8].tolist()], "flags", int(flags.max()))


if __name__ == "__main__":
    main()
