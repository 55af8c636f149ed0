"""M-AVG of learners with normalised residual blocks, on textured images: group norm, dropout and the meta step of the library, put
together by autograd.

A learner's net on images of S positions, channels last (patches: the 3x3 neighbourhoods of the pixels):
    h = patches W_0
    h = h + dropout(silu(group_norm(h)) W_t)            for every block t
    logits = mean over positions(silu(group_norm(h))) W_head + b_head
All P learners are one batch: activations [P][B][S][C], every weight [P][..], a learner's weights together in its row of the
replicas [P][n], which the meta step reads.  Weight products are torch's, in the type of the activations.

  python -m paper_2110_00625_amd.residual --P 8 --rounds 20
"""
import argparse

import numpy as np
import torch

from . import kavg, layers, synth


class _Product(torch.autograd.Function):
    """x [P][M][c_in] times weight [P][c_in][c_out] in x's type; weight and its gradient in float32."""

    @staticmethod
    def forward(ctx, x, weight):
        w = weight.to(x.dtype)
        ctx.save_for_backward(x, w)
        return torch.bmm(x, w)

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        dy = dy.contiguous()
        dx = torch.bmm(dy, w.transpose(1, 2).contiguous()) if ctx.needs_input_grad[0] else None
        return dx, torch.bmm(x.transpose(1, 2).contiguous(), dy).float()


def patches(X, dtype):
    """[N][H][W][c] -> [N][H*W][9c]: the pixels' 3x3 neighbourhoods, the image continued around its edges."""
    N, H, W, _ = X.shape
    shifted = [torch.roll(X, (1 - kh, 1 - kw), (1, 2)) for kh in range(3) for kw in range(3)]
    return torch.cat(shifted, 3).reshape(N, H * W, -1).to(dtype)


class ResidualLearners:
    def __init__(self, P, c_in, channels, blocks, groups, classes, lr, mu, drop=0.1, seed=0, dtype=torch.bfloat16, device="cuda"):
        self.P, self.blocks, self.groups, self.lr, self.mu, self.drop, self.seed = P, blocks, groups, lr, mu, drop, seed
        self.dtype, self.step = dtype, 0
        shapes = [("w0", (c_in, channels))]
        for t in range(blocks):
            shapes += [("gamma%d" % t, (channels,)), ("beta%d" % t, (channels,)), ("w%d" % (t + 1), (channels, channels))]
        shapes += [("gamma", (channels,)), ("beta", (channels,)), ("head", (channels, classes)), ("b", (classes,))]
        start, rng = [], np.random.default_rng(seed)
        for name, shape in shapes:
            if name.startswith("gamma"):
                start.append(np.ones(shape, np.float32))
            elif len(shape) == 1:
                start.append(np.zeros(shape, np.float32))
            else:
                start.append(rng.standard_normal(shape, dtype=np.float32) * np.float32(shape[0] ** -0.5))
        self.w = torch.from_numpy(np.concatenate([a.ravel() for a in start])).to(device)
        self.v = torch.zeros_like(self.w)
        self.replicas = self.w.repeat(P, 1)
        self.params, at = {}, 0
        for name, shape in shapes:
            n = int(np.prod(shape))
            self.params[name] = self.replicas[:, at:at + n].view(P, *shape)          # (a learner's part of its row)
            at += n

    def losses(self, params, x, y):
        """Mean loss of every learner [P] on its own batch: x [P][B][S][c_in], y [P][B]."""
        P, B, S, _ = x.shape

        def product(h, w):
            return _Product.apply(h.reshape(P, B * S, -1), w).view(P, B, S, -1)
        h = product(x.to(self.dtype), params["w0"])
        for t in range(self.blocks):
            a = layers.group_norm(h, params["gamma%d" % t], params["beta%d" % t], self.groups, activation="silu")
            # (a learner's mask is its part of the one mask of the batch; every step has a seed, every block a site of its own)
            h = layers.dropout(product(a, params["w%d" % (t + 1)]), self.drop, self.seed + self.step, site=t, residual=h)
        a = layers.group_norm(h, params["gamma"], params["beta"], self.groups, activation="silu")
        logits = torch.bmm(a.float().mean(2), params["head"]) + params["b"][:, None]
        return -torch.log_softmax(logits, 2).gather(2, y[:, :, None].long()).mean((1, 2))

    def gradients(self, x, y):
        """(losses [P], gradient of every parameter)."""
        leaves = {k: p.detach().requires_grad_() for k, p in self.params.items()}
        losses = self.losses(leaves, x, y)
        return losses.detach(), torch.autograd.grad(losses.sum(), list(leaves.values()))

    def local_step(self, x, y):
        losses, grads = self.gradients(x, y)
        torch._foreach_add_(list(self.params.values()), list(grads), alpha=-self.lr)
        self.step += 1
        return losses

    def meta_update(self):
        """Average of the replicas, block momentum, restart of the learners."""
        kavg.kavg_meta_update_flat(self.w, self.v, self.replicas, self.mu)


def train(P=8, K=4, B=32, side=16, channels=64, blocks=2, groups=8, classes=10, lr=0.1, mu=0.5, drop=0.1, rounds=20, N=2048, seed=7,
          dtype=torch.bfloat16, quiet=True):
    """Mean training loss of every round."""
    data = synth.make_image_dataset(N, side, side, 3, 8, classes, seed_data=seed, seed_texture=seed + 1)
    X = patches(torch.from_numpy(data["X32"]).cuda().view(N, side, side, 8)[..., :3], dtype)
    y = torch.from_numpy(data["y"]).cuda()
    net = ResidualLearners(P, X.shape[2], channels, blocks, groups, classes, lr, mu, drop, seed, dtype)
    rng, curve = np.random.default_rng(seed + 2), []
    for r in range(rounds):
        total = 0.
        for _ in range(K):
            idx = torch.from_numpy(rng.integers(0, N, (P, B))).cuda()
            total += net.local_step(X[idx], y[idx]).mean()
        net.meta_update()
        curve.append(float(total) / K)
        if not quiet:
            print("round %3d  loss %.4f" % (r, curve[-1]), flush=True)
    return curve


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("P", 8), ("K", 4), ("B", 32), ("side", 16), ("channels", 64), ("blocks", 2), ("groups", 8), ("rounds", 20),
                          ("N", 2048), ("seed", 7)):
        ap.add_argument("--" + name, type=int, default=default)
    for name, default in (("lr", 0.1), ("mu", 0.5), ("drop", 0.1)):
        ap.add_argument("--" + name, type=float, default=default)
    ap.add_argument("--f32", action="store_true", help="activations in float32")
    a = vars(ap.parse_args())
    train(dtype=torch.float32 if a.pop("f32") else torch.bfloat16, quiet=False, **a)


if __name__ == "__main__":
    main()
