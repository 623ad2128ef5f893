"""Experts that are no DC-CGANs, one for each label, on the library's operators: a denoiser of digit-like images.

    python examples/label_experts.py [steps]

A batch of mixed labels is sorted by label; every label's rows then go through weights of its own:

    h = x W_in              group_linear
    s = h + norm(h) W_mid   rms_norm, group_linear; the sum is formed by the next norm
    y = norm(s) W_out       rms_norm with the residual's addition, group_linear

Training is in bf16 with fp32 weights: the gradients are group_linear_dgrad, group_linear_wgrad and rms_norm_backward, and one AdamW step with 8-bit moments
updates all tensors and writes the bf16 copies that the products read.  Serving is in 8 bits: the weights are quantized once, the norms write the operands of
the 8-bit products."""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2102_10485_amd import BF16, FP32, binding, synth  # noqa: E402

LABELS, SIDE, WIDE, EPS = 10, 28, 512, 1e-5
PIXELS = SIDE * SIDE


def batch(n, seed):
    """Images of random labels, sorted by label: (clean, noisy), and where each label's rows start."""
    rng = np.random.default_rng(seed)
    label = rng.integers(0, LABELS, n)
    label = label[np.argsort(label, kind="stable")]
    clean = synth.blob_images(label, rng, SIDE, LABELS).reshape(n, PIXELS)
    noisy = clean + rng.normal(0, 0.5, clean.shape)
    offs = np.searchsorted(label, np.arange(LABELS + 1)).astype(np.int32)
    return torch.from_numpy(clean).cuda(), torch.from_numpy(noisy).cuda().bfloat16(), torch.from_numpy(offs).cuda()


class Experts:
    SHAPES = dict(w_in=(LABELS, WIDE, PIXELS), w_mid=(LABELS, WIDE, WIDE), w_out=(LABELS, PIXELS, WIDE), gain_mid=(WIDE,), gain_out=(WIDE,))

    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.p = {k: torch.ones(s, device="cuda") if k.startswith("gain") else torch.randn(s, generator=gen, device="cuda") * s[-1] ** -0.5 for k, s in self.SHAPES.items()}
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.w = {k: v.bfloat16() for k, v in self.p.items()}                    # what the products read
        sizes = [v.numel() for v in self.p.values()]
        blocks = binding.adamw_blocks(sizes)
        self.moments = [torch.zeros(blocks * 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scales = [torch.zeros(blocks, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.optimizer = binding.AdamW(sizes, [v.data_ptr() for v in self.p.values()], [v.data_ptr() for v in self.g.values()], FP32,
                                       [v.data_ptr() for v in self.w.values()], [0.0 if k.startswith("gain") else 0.01 for k in self.p], 8,
                                       *(v.data_ptr() for v in self.moments + self.scales))
        self.t = 0

    # the operators on tensors
    def linear(self, x, name, offs):
        _, n_out, n_in = self.SHAPES[name]
        y = torch.empty((len(x), n_out), dtype=torch.bfloat16, device="cuda")
        binding.group_linear(BF16, x.data_ptr(), n_in, self.w[name].data_ptr(), offs.data_ptr(), LABELS, len(x), n_in, n_out, y.data_ptr(), n_out, stream())
        return y

    def linear_backward(self, x, dy, name, offs, want_dx=True):
        _, n_out, n_in = self.SHAPES[name]
        nbytes = binding.group_linear_wgrad_bytes(LABELS, len(x), n_in, n_out)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        binding.group_linear_wgrad(BF16, x.data_ptr(), n_in, dy.data_ptr(), n_out, offs.data_ptr(), LABELS, len(x), n_in, n_out, self.g[name].data_ptr(),
                                   work.data_ptr(), nbytes, stream())
        if want_dx:
            dx = torch.empty((len(x), n_in), dtype=torch.bfloat16, device="cuda")
            binding.group_linear_dgrad(BF16, dy.data_ptr(), n_out, self.w[name].data_ptr(), offs.data_ptr(), LABELS, len(x), n_in, n_out, dx.data_ptr(), n_in, stream())
            return dx

    def norm(self, x, residual, name):
        rows = len(x)
        total = torch.empty_like(x) if residual is not None else x
        y, inv = torch.empty_like(x), torch.empty(rows, device="cuda")
        binding.rms_norm(BF16, x.data_ptr(), WIDE, residual.data_ptr() if residual is not None else 0, WIDE, self.p[name].data_ptr(), EPS, rows, WIDE,
                         total.data_ptr() if residual is not None else 0, WIDE, y.data_ptr(), WIDE, 0, 0, inv.data_ptr(), stream())
        return total, y, inv

    def norm_backward(self, dy, total, inv, dtotal, name):
        dx, nbytes = torch.empty_like(dy), binding.rms_norm_backward_bytes(len(dy), WIDE)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        binding.rms_norm_backward(BF16, dy.data_ptr(), WIDE, total.data_ptr(), WIDE, self.p[name].data_ptr(), inv.data_ptr(), dtotal.data_ptr() if dtotal is not None else 0,
                                  WIDE, len(dy), WIDE, dx.data_ptr(), WIDE, self.g[name].data_ptr(), work.data_ptr(), nbytes, stream())
        return dx

    def forward(self, x, offs):
        h = self.linear(x, "w_in", offs)
        _, n1, inv1 = self.norm(h, None, "gain_mid")
        s, n2, inv2 = self.norm(self.linear(n1, "w_mid", offs), h, "gain_out")
        return self.linear(n2, "w_out", offs), (h, n1, inv1, s, n2, inv2)

    def train_step(self, clean, noisy, offs, lr=1e-3):
        y, (h, n1, inv1, s, n2, inv2) = self.forward(noisy, offs)
        off = y.float() - clean
        dy = (off * (2.0 / off.numel())).bfloat16()
        dn2 = self.linear_backward(n2, dy, "w_out", offs)
        ds = self.norm_backward(dn2, s, inv2, None, "gain_out")                  # the gradient of both terms of the sum
        dn1 = self.linear_backward(n1, ds, "w_mid", offs)
        dh = self.norm_backward(dn1, h, inv1, ds, "gain_mid")
        self.linear_backward(noisy, dh, "w_in", offs, want_dx=False)
        self.t += 1
        self.optimizer.step(lr, 0.9, 0.999, 1e-8, self.t, 1, stream())
        return (off * off).mean()

    # serving in 8 bits
    def quantized(self, x, precision=BF16):
        """(codes, scales) of a matrix, or of every expert's."""
        cols = x.shape[-1]
        wide = -(-cols // 128) * 128
        q = torch.empty((*x.shape[:-1], wide), dtype=torch.uint8, device="cuda")
        scale = torch.empty((*x.shape[:-1], wide // 128), dtype=torch.uint8, device="cuda")
        binding.quantize8(precision, x.data_ptr(), cols, x.numel() // cols, cols, q.data_ptr(), scale.data_ptr(), stream())
        return q, scale

    def freeze(self):
        self.w8 = {k: self.quantized(v, FP32) for k, v in self.p.items() if k.startswith("w")}

    def linear8(self, x8, name, offs):
        _, n_out, n_in = self.SHAPES[name]
        y = torch.empty((len(x8[0]), n_out), dtype=torch.bfloat16, device="cuda")
        binding.group_linear8(*(v.data_ptr() for v in x8 + self.w8[name]), offs.data_ptr(), LABELS, len(y), n_in, n_out, BF16, y.data_ptr(), n_out, stream())
        return y

    def norm8(self, x, residual, name):
        q, scale = (torch.empty((len(x), w), dtype=torch.uint8, device="cuda") for w in (WIDE, WIDE // 128))
        binding.rms_norm(BF16, x.data_ptr(), WIDE, residual.data_ptr() if residual is not None else 0, WIDE, self.p[name].data_ptr(), EPS, len(x), WIDE,
                         0, 0, 0, 0, q.data_ptr(), scale.data_ptr(), 0, stream())
        return q, scale

    def serve(self, x, offs):
        h = self.linear8(self.quantized(x), "w_in", offs)
        return self.linear8(self.norm8(self.linear8(self.norm8(h, None, "gain_mid"), "w_mid", offs), h, "gain_out"), "w_out", offs)


def stream():
    return torch.cuda.current_stream().cuda_stream


def main(steps=200, n=1280):
    torch.cuda.set_device(0)
    experts, losses = Experts(), []
    for k in range(steps):
        losses.append(experts.train_step(*batch(n, k)))
    losses = [float(v) for v in losses]
    clean, noisy, offs = batch(64, 10 ** 6)
    experts.freeze()
    exact, served = experts.forward(noisy, offs)[0].float(), experts.serve(noisy, offs).float()
    error, noise = float(((served - clean) ** 2).mean()), float(((noisy.float() - clean) ** 2).mean())
    print("squared error: %.4f before training, %.4f after %d steps, %.4f served in 8 bits (of the noisy images: %.4f); 8-bit outputs differ by %.3f of their norm"
          % (losses[0], losses[-1], steps, error, noise, float((served - exact).norm() / exact.norm())))
    return losses, error, noise, float((served - exact).norm() / exact.norm())


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
