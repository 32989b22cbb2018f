"""Embeddings held as microscaled 4-bit rows, beside a graph over the rows themselves:

  the exact neighbours among the 4-bit rows, and how many of them the graph's search finds
  the scores of a batch of questions against all rows, and one row drawn for each of them by its score

    python examples/draw_neighbours.py [--n 100000] [--d 128] [--nq 256] [--k 10]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2305_04359_amd import binding as ann  # noqa: E402


def embeddings(n, d, generator, centres):
    x = centres[torch.randint(0, len(centres), (n,), device="cuda", generator=generator)]
    x = x + 0.1 * torch.randn((n, d), device="cuda", generator=generator)
    return x / x.norm(dim=1, keepdim=True)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--n", type=int, default=100_000)
    p.add_argument("--d", type=int, default=128)
    p.add_argument("--nq", type=int, default=256)
    p.add_argument("--k", type=int, default=10)
    p.add_argument("--seed", type=int, default=1)
    o = p.parse_args(argv)
    g = torch.Generator(device="cuda")
    g.manual_seed(o.seed)
    centres = torch.randn((64, o.d), device="cuda", generator=g) / o.d ** 0.5
    points, questions = embeddings(o.n, o.d, g, centres), embeddings(o.nq, o.d, g, centres)

    rows = ann.ann_mx_quantize(points, norms=True)
    exact, _ = ann.ann_mx_search(rows, ann.ann_mx_quantize(questions, norms=True), o.k)
    graph = ann.ann_build(points, R=32, L=64, alpha=1.2)
    found, _ = ann.ann_search(graph, points, questions, k=o.k, L=4 * o.k)
    recall = (exact.long().unsqueeze(2) == found.long().unsqueeze(1)).any(2).float().mean().item()

    scores = ann.ann_mx_product(questions, rows)
    uniform = torch.rand(o.nq, device="cuda", generator=g)
    drawn, logprobs = ann.ann_sample(scores, uniform, temperature=0.02, top_k=o.k, top_p=0.95)
    near = scores.gather(1, drawn.long().unsqueeze(1)).mean().item()

    held = rows.codes.numel() + rows.scales.numel()
    print(f"{o.n} rows of {o.d}: {points.numel() * 4 / 2 ** 20:.1f} MiB as float32, {held / 2 ** 20:.1f} MiB as 4-bit rows")
    print(f"neighbours among the 4-bit rows that the graph over the float rows finds: {recall:.3f}")
    print(f"drawn rows: mean score {near:.3f} (all rows {scores.mean().item():.3f}), mean log-probability {logprobs.mean().item():.2f}")
    return recall, near, drawn, logprobs, scores


if __name__ == "__main__":
    main()
