"""From segmentation output to a trained per-bird encoder.

    python examples/bird_encoder.py [--steps 60]

Probability maps of a few frames become detections (mask_components_frames),
the detections' places are clustered (cluster_frames), and an encoder that
sees nothing but the detections learns to tell which birds are core, border
and noise, by attention among the birds of a frame: layer_norm_rows,
rotary_frames and attention_frames with their gradients, on the CSR batch
that the detections come in.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2512_07009_amd as flock  # noqa: E402
from paper_2512_07009_amd import encoder, workloads  # noqa: E402


def detections(seed, frames, height, width, n_birds):
    """Detections of synthetic probability maps: xy, offsets, features [T, 6]."""
    prob = torch.from_numpy(workloads.bird_masks(seed, frames, height, width, n_birds=n_birds)).cuda()
    det = flock.mask_components_frames(prob, 0.5, 8, with_labels=False)
    total = int(det["offsets"][-1])
    box = det["box"][:total].float()
    size = torch.tensor([width, height], device="cuda")
    features = torch.cat([det["centroid"][:total].float() / size, box[:, 2:] / 16,
                          torch.log1p(det["area"][:total].float())[:, None], det["score"][:total, None]], 1)
    return det["xy"][:total].contiguous(), det["offsets"], features


def main(steps=60, frames=8, height=360, width=640, n_birds=300, features=128, seed=0, quiet=False):
    torch.manual_seed(seed)
    xy, offsets, detected = detections(seed, frames, height, width, n_birds)
    _, kind, _ = flock.cluster_frames(xy, offsets, eps_px=35.0, min_pts=4)
    target = kind.long()

    waves = [2 * torch.pi / (16.0 * 2 ** j) for j in range(8)]     # 16 px to 2048 px
    block = encoder.EncoderBlock(features, q_heads=4, kv_heads=2, head_dim=64, sigma_px=(10.0, 200.0),
                                 axes=flock.RotaryAxes(y=waves, x=waves)).cuda()
    embed = torch.nn.Linear(detected.shape[1], features).cuda()
    classify = torch.nn.Linear(features, 3).cuda()
    optimizer = torch.optim.AdamW([*block.parameters(), *embed.parameters(), *classify.parameters()], lr=1e-3)
    losses = []
    for step in range(steps):
        h = block(embed(detected).to(torch.bfloat16), offsets, xy)
        scores = classify(h.float())
        loss = torch.nn.functional.cross_entropy(scores, target)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).cpu()
    right = (scores.argmax(1) == target).float().mean().item()
    if not quiet:
        share = torch.bincount(target, minlength=3).float() / len(target)
        print(f"{len(target)} detections in {frames} frames (noise, border, core: "
              f"{', '.join(f'{s:.2f}' for s in share.tolist())})")
        print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps, {right:.1%} of the birds told apart")
    return losses, right


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=60)
    main(parser.parse_args().steps)
