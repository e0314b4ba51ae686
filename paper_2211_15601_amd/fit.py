"""Learn a skinning field from points whose canonical places are known: the correspondence search, its backward, and the clipped AdamW
step in one training loop.

    python -m paper_2211_15601_amd.fit --steps 100

The weight grid is a softmax over the bones of a grid of logits (as the paper's skinning network ends); each pose's bones also get a
learned shift, as where poses come from an estimate.  Every step poses a batch of points with the true field, searches their canonical
correspondences with the learned one, and pulls the nearest root of each point to where the point came from.  A root near a fold has a
large inverse Jacobian and a gradient to match: hence the limit on the global norm, which the step applies by itself, and one on each pose's shift
before that, so that a pose that is off takes nothing from the field."""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding, optim, workloads as wl
from .autograd import CorrespondenceSearch


def poses(seed, dims, n_points, n_poses):
    """The true weight grid, and [(bones [1,n_b,12], posed points [3,N], canonical points [3,N])] on the GPU."""
    rng = np.random.default_rng(seed)
    a, b = wl.random_segments(rng)
    up = lambda v: torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()
    out = []
    for _ in range(n_poses):
        B = wl.independent_bone_transforms(rng, wl.N_BONES)
        x = rng.uniform(wl.BOX_LO.astype(np.float64), wl.BOX_HI.astype(np.float64), size=(n_points, 3))
        out.append((up(B[None]), up(wl.pose_points(x, a, b, B).T), up(x.T)))
    return up(wl.weight_grid(dims, a, b)), out


def train(steps=100, dims=(16, 16, 4), n_points=4096, n_poses=4, lr=0.05, max_norm=0.01, shift_norm=0.01, seed=0):
    """Returns the losses (mean squared distance of the nearest roots), the gradients' norms, their largest entries, and the optimizer."""
    W_true, data = poses(seed, dims, n_points, n_poses)
    logits = (0.25 * (W_true + 1e-4).log()).requires_grad_(True)          # a field that is far too smooth
    shift = [torch.zeros(wl.N_BONES, 3, device="cuda", requires_grad=True) for _ in data]
    params = [logits, *shift]
    for p in params:                                                       # gradients stay where they are: backward adds, zero_grad clears
        p.grad = torch.zeros_like(p)
    grads, shift_grads = optim.TensorList([p.grad for p in params]), [optim.TensorList([s.grad]) for s in shift]
    fs = binding.Context(dims, wl.N_BONES, wl.BOX_LO, wl.BOX_HI)
    # the shifts go by a fraction of the rate and do not decay; a batch that spoils the gradients is left out
    opt = optim.AdamW(params, lr=lr, weight_decay=0.0, max_norm=max_norm, skip_nonfinite=True,
                      lr_scales=[1.0] + [0.02] * n_poses, decay_scales=[1.0] + [0.0] * n_poses)
    losses, norms, peaks = [], [], []
    for step in range(steps):
        p = step % n_poses
        B, xq, x = data[p]
        W = torch.softmax(logits, dim=-1)
        moved = torch.cat([B.view(wl.N_BONES, 3, 4)[..., :3], B.view(wl.N_BONES, 3, 4)[..., 3:] + shift[p][..., None]], dim=-1)
        roots, conv = CorrespondenceSearch.apply(fs, W, moved.reshape(1, wl.N_BONES, 12), xq, None)
        far = ((roots - x) ** 2).sum(1).masked_fill(conv == 0, torch.inf)  # [K,N]
        nearest = far.amin(0)
        found = nearest < torch.inf
        loss = nearest.masked_fill(~found, 0.0).sum() / found.sum().clamp_min(1)
        loss.backward()
        peaks.append(grads.grad_norm(kind="max"))
        shift_grads[p].clip_grads(shift_norm)
        norms.append(opt.step())
        opt.zero_grad()
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), torch.cat(norms).tolist(), torch.cat(peaks).tolist(), opt


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--points", type=int, default=4096)
    ap.add_argument("--max-norm", type=float, default=0.01)
    args = ap.parse_args()
    losses, norms, peaks, opt = train(args.steps, n_points=args.points, max_norm=args.max_norm)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:4d}: loss {losses[i]:.3e}, gradient norm {norms[i]:.3e}, largest {peaks[i]:.3e}")
    print(f"last: loss {losses[-1]:.3e}; {sum(n > args.max_norm for n in norms)} of {len(norms)} steps clipped, {int(opt.step_count)} taken")


if __name__ == "__main__":
    main()
