"""Personalise a shared head for many sites, and serve certified answers with it.

A proxy keeps one head W [C, d] for all sites and a low-rank pair (A_s, B_s) for
each.  Every site names the classes its own way, here by a swap of some labels.

  train   batches mix requests of all sites: ``adapter_forward`` gives their
          logits in one call, ``adapter_backward`` the gradients of every pair,
          ``muon_step`` moves all factors along their orthogonalised momentum
  serve   single queries of different sites in one ``adapter_forward``
  cache   a site's own head W + scale B A certifies and fills a cache of its own;
          a step on W itself moves sigma_max(W) by a bounded amount (float32 here: up to W's rounding)

    python examples/adapt_sites.py [--sites 16] [--steps 60]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2608_13144_amd import api  # noqa: E402

MOST = 1.21  # the largest singular value that a step's update can have


def requests(rows: list[int], sites: list[int], device) -> tuple[torch.Tensor, torch.Tensor]:
    """Offsets and pairs of one batch: request i has rows[i] rows of site sites[i]."""
    offsets = [0]
    for n in rows:
        offsets.append(offsets[-1] + n)
    return (torch.tensor(offsets, dtype=torch.int32, device=device),
            torch.tensor(sites, dtype=torch.int32, device=device))


def run(sites: int = 16, d: int = 256, C: int = 200, r: int = 8, rows: int = 64, steps: int = 60, lr: float = 0.1,
        seed: int = 0, device: str = "cuda:0") -> dict:
    g = torch.Generator(device=device).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=device)
    # features around one centre a class; the shared head knows them, the sites swap a few classes
    centres = 2.0 * randn(C, d) / math.sqrt(d)
    W = 1.5 * centres
    bias = torch.zeros(C, device=device)
    swaps = torch.arange(C, device=device).repeat(sites, 1)
    for s in range(sites):
        a, b = torch.randperm(C, generator=g, device=device)[:2].tolist()
        swaps[s, a], swaps[s, b] = b, a
    A = randn(sites, r, d) / math.sqrt(d)
    B = torch.zeros(sites, C, r, device=device)
    scale = torch.ones(sites, device=device)
    MA, MB = torch.zeros_like(A), torch.zeros_like(B)
    offsets, adapter = requests([rows] * sites, list(range(sites)), device)
    site = torch.arange(sites, device=device).repeat_interleave(rows)

    def batch():
        # one row in four from the classes that its site swaps
        label = torch.randint(0, C, (sites * rows,), generator=g, device=device)
        odd = (swaps != torch.arange(C, device=device)).float().argmax(1)
        pick = torch.rand(sites * rows, generator=g, device=device) < 0.25
        label = torch.where(pick, odd[site], label)
        x = centres[label] + 0.3 * randn(sites * rows, d) / math.sqrt(d)
        return x, swaps[site, label]

    losses = []
    for step in range(steps):
        x, y = batch()
        out = api.adapter_forward(x, W, bias, A, B, scale, offsets, adapter, keep=True)
        log_p = torch.log_softmax(out.y, 1)
        losses.append(-log_p.gather(1, y[:, None]).mean())
        dy = log_p.exp()
        dy.scatter_add_(1, y[:, None], torch.full_like(dy[:, :1], -1.0))
        dy /= rows
        grad = api.adapter_backward(dy, x, W, A, B, scale, offsets, adapter, v=out.v, want_dx=False)
        rate = lr * (1.0 - step / steps)
        api.muon_step(A, grad.dA, MA, rate)
        api.muon_step(B, grad.dB, MB, rate)

    # one query of each site at a time, all in one call
    x, _ = batch()
    queries = x[::rows].contiguous()
    single = requests([1] * sites, list(range(sites)), device)
    logits = api.adapter_forward(queries, W, bias, A, B, scale, *single).y

    # site 0's own head certifies its features and answers from a cache of its own
    W0 = torch.addmm(W, B[0], A[0], alpha=float(scale[0]))
    sigma0 = api.spectral_norm(W0).sigma
    z = x[:rows].contiguous()
    cert = api.certify(z, W0, bias, sigma0)
    cache = api.LipCache(d, rows, device=device)
    cache.insert(z, cert.label, cert.r)
    answers = cache.lookup(z)
    agree, hits = (answers.label == cert.label) & (answers.label >= 0), answers.label >= 0

    # a step on the shared head: its spectral norm moves by at most MOST lr scale (no decay here) and W's rounding
    before = api.spectral_norm(W).sigma
    x, y = batch()
    p = torch.softmax(api.adapter_forward(x, W, bias, A, B, scale, offsets, adapter).y, 1)
    p.scatter_add_(1, y[:, None], torch.full_like(p[:, :1], -1.0))
    moved, M = W.clone(), torch.zeros_like(W)
    api.muon_step(moved, (p.t() @ x) / len(x), M, lr)
    after = api.spectral_norm(moved).sigma
    return dict(first=float(losses[0]), last=float(torch.stack(losses[-5:]).mean()), logits=logits, queries=queries,
                W=W, A=A, B=B, scale=scale, hits=int(hits.sum()), agree=int(agree.sum()), rows=rows,
                certified=int((cert.r > 0).sum()), moved=abs(after - before),
                bound=MOST * lr * max(1.0, C / d) ** 0.5)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sites", type=int, default=16)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    out = run(sites=a.sites, steps=a.steps)
    print(f"loss {out['first']:.3f} -> {out['last']:.3f} over {a.steps} steps on {a.sites} sites")
    print(f"site 0: {out['certified']} of {out['rows']} features certified, {out['hits']} found, {out['agree']} with their label")
    print(f"a step on the shared head moved sigma_max by {out['moved']:.4f} (bound {out['bound']:.4f})")


if __name__ == "__main__":
    main()
