"""Trains a ResidualMLP on synthetic data: RMS norms with 8-bit codes, 8-bit products with GELU, binary
projections with the 1-bit FQT backward, Muon for the weight matrices and Adam for the rest.

  python examples/train_residual_mlp.py [--steps 60] [--batch 512] [--operands int8|e4m3|bf16]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2408_14267_amd import blocks, train  # noqa: E402


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=512)
    ap.add_argument("--operands", choices=("int8", "e4m3", "bf16"), default="int8")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    features, classes = 128, 10
    model = blocks.ResidualMLP(features, classes, operands=a.operands).cuda()
    opt = blocks.muon_and_adam(model, first_last=(model.stem, model.head))
    centres = torch.randn(classes, features, device="cuda")
    losses = []
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for step in range(a.steps):
        y = torch.randint(classes, (a.batch,), device="cuda")
        x = centres[y] + 1.5 * torch.randn(a.batch, features, device="cuda")
        losses.append(train.train_step(model, opt, x, y))
        if step % 10 == 0 or step + 1 == a.steps:
            print(f"step {step:4d}  loss {losses[-1].item():.4f}", flush=True)
    torch.cuda.synchronize()
    print(f"{(time.perf_counter() - begin) / a.steps * 1e3:.2f} ms a step")
    return [v.item() for v in losses]


if __name__ == "__main__":
    main()
