"""Experts that rows choose themselves, on the library's operators: a denoiser of digit-like images whose labels are not known.

    python examples/routed_experts.py [steps]

    h = gelu(x W_in + b_in)                          group_linear_act, of one expert
    n = norm(h)                                      rms_norm
    every row goes to two of sixteen experts:        group_linear (the logits n W_gate), route, sort_by_label, gather_rows
        o = gelu(n W_up[e] + b_up[e]) W_down[e] + b_down[e]          group_linear_act, twice
    s = h + dropout(sum of weight * o)               combine_rows, dropout
    y = s W_out + b_out                              group_linear_act

Training is in bf16 with fp32 weights, with the balance loss beside the squared error; nothing of a step leaves the device, and its gradients may be captured into a graph.  Serving is in 8 bits,
without dropout: the weights are quantized once."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2102_10485_amd import BF16, FP32, binding as B, synth  # noqa: E402

import numpy as np  # noqa: E402

EXPERTS, K, SIDE, WIDE, HIDDEN, EPS, DROP, BALANCE, SEED = 16, 2, 28, 512, 768, 1e-5, 0.1, 0.01, 2024
PIXELS = SIDE * SIDE


def batch(n, seed):
    """Images of random labels, clean and noisy."""
    rng = np.random.default_rng(seed)
    clean = synth.blob_images(rng.integers(0, 10, n), rng, SIDE, 10).reshape(n, PIXELS)
    noisy = clean + rng.normal(0, 0.5, clean.shape)
    return torch.from_numpy(clean).cuda(), torch.from_numpy(noisy).cuda().bfloat16()


def stream():
    return torch.cuda.current_stream().cuda_stream


def at(t):
    return 0 if t is None else t.data_ptr()


def new(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


class Denoiser:
    # experts, outputs, inputs
    SHAPES = dict(w_in=(1, WIDE, PIXELS), w_gate=(1, EXPERTS, WIDE), w_up=(EXPERTS, HIDDEN, WIDE), w_down=(EXPERTS, WIDE, HIDDEN), w_out=(1, PIXELS, WIDE))
    BIASES = dict(b_in=(1, WIDE), b_up=(EXPERTS, HIDDEN), b_down=(EXPERTS, WIDE), b_out=(1, PIXELS))

    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.p = {k: torch.randn(s, generator=gen, device="cuda") * s[-1] ** -0.5 for k, s in self.SHAPES.items()}
        self.p.update({k: torch.zeros(s, device="cuda") for k, s in self.BIASES.items()}, gain=torch.ones(WIDE, device="cuda"))
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.w = {k: v.bfloat16() for k, v in self.p.items()}                    # what the products read
        sizes = [v.numel() for v in self.p.values()]
        blocks = B.adamw_blocks(sizes)
        self.moments = [torch.zeros(blocks * 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scales = [torch.zeros(blocks, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.optimizer = B.AdamW(sizes, [v.data_ptr() for v in self.p.values()], [v.data_ptr() for v in self.g.values()], FP32, [v.data_ptr() for v in self.w.values()],
                                 [0.01 if k.startswith("w") else 0.0 for k in self.p], 8, *(v.data_ptr() for v in self.moments + self.scales))
        self.t = 0
        self.step_on_device = torch.zeros(1, dtype=torch.int32, device="cuda")   # what dropout counts: a captured step moves it on itself

    # the operators on tensors
    def linear(self, x, name, bias, offs, act=B.ACT_NONE, store_z=False):
        _, n_out, n_in = self.SHAPES[name]
        y, z = new(len(x), n_out), new(len(x), n_out) if store_z else None
        B.group_linear_act(BF16, at(x), n_in, at(self.w[name]), at(offs), self.SHAPES[name][0], len(x), n_in, n_out, at(self.p[bias]) if bias else 0, act, 0, 0, at(z), n_out, at(y),
                           n_out, stream())
        return (y, z) if store_z else y

    def gradients(self, x, dz, name, bias, offs):
        """Those of a product's weights and bias from the gradient of its sums."""
        groups, n_out, n_in = self.SHAPES[name]
        n = B.group_linear_wgrad_bytes(groups, len(x), n_in, n_out)
        B.group_linear_wgrad(BF16, at(x), n_in, at(dz), n_out, at(offs), groups, len(x), n_in, n_out, at(self.g[name]), at(new(n, dtype=torch.uint8)), n, stream())
        if bias:
            self.through(dz, None, bias, offs, B.ACT_NONE, False)

    def through(self, dy, z, bias, offs, act, want_dz=True):
        """The gradient through an activation, and the bias's."""
        groups, cols = self.BIASES[bias]
        n = B.group_act_backward_bytes(groups, len(dy), cols)
        dz = torch.empty_like(dy) if want_dz else None
        B.group_act_backward(BF16, at(dy), cols, act, at(z), cols, at(offs), groups, len(dy), cols, at(dz), cols, at(self.g[bias]), at(new(n, dtype=torch.uint8)), n, stream())
        return dz

    def back(self, dz, name, offs, other=None, act=B.ACT_NONE, z=None):
        """The gradient of a product's inputs, or of the sums whose activation they were."""
        groups, n_out, n_in = self.SHAPES[name]
        dx = new(len(dz), n_in)
        B.group_linear_dgrad_act(BF16, at(dz), n_out, at(self.w[name]), at(offs), groups, len(dz), n_in, n_out, at(other), n_in, act, at(z), n_in, at(dx), n_in, stream())
        return dx

    def choose(self, logits, train):
        """Experts, weights, what the gradient needs, and the rows' places."""
        n, i32 = len(logits), torch.int32
        expert, weight = new(n, K, dtype=i32), new(n, K, dtype=torch.float32)
        counts, balance = (new(EXPERTS + 1, dtype=i32), new(1, dtype=torch.float32)) if train else (None, None)
        size = B.route_bytes(n, EXPERTS) if train else 0
        B.route(BF16, at(logits), EXPERTS, n, EXPERTS, K, True, at(expert), at(weight), at(counts), 0, at(balance), at(new(size, dtype=torch.uint8)), size, stream())
        offs, place, size = new(EXPERTS + 1, dtype=i32), new(n, K, dtype=i32), B.sort_by_label_bytes(n * K, EXPERTS)
        B.sort_by_label(at(expert), n * K, EXPERTS, at(offs), 0, at(place), at(new(size, dtype=torch.uint8)), size, stream())
        return expert, weight, counts, balance, offs, place

    def hand_out(self, x, place, offs):
        xs = new(len(x) * K, WIDE)
        B.gather_rows(BF16, at(x), WIDE, at(place), at(offs), EXPERTS, K, len(x), WIDE, at(xs), WIDE, stream())
        return xs

    def together(self, o, place, weight, offs, residual=None):
        y = new(len(place), WIDE)
        B.combine_rows(BF16, at(o), WIDE, at(place), at(weight), at(offs), EXPERTS, K, at(residual), WIDE, len(place), WIDE, at(y), WIDE, stream())
        return y

    def dropout(self, x, residual):
        y = torch.empty_like(x)
        B.dropout(BF16, at(x), WIDE, at(residual), WIDE, len(x), WIDE, DROP, SEED, 0, 0, at(self.step_on_device), at(y), WIDE, stream())
        return y

    def norm(self, x):
        y, inv = torch.empty_like(x), new(len(x), dtype=torch.float32)
        B.rms_norm(BF16, at(x), WIDE, 0, 0, at(self.p["gain"]), EPS, len(x), WIDE, 0, 0, at(y), WIDE, 0, 0, at(inv), stream())
        return y, inv

    def forward(self, x, train=True):
        one = torch.zeros(2, dtype=torch.int32, device="cuda")
        one[1:] = len(x)
        h, z_in = self.linear(x, "w_in", "b_in", one, B.ACT_GELU, True)
        n, inv = self.norm(h)
        logits = self.linear(n, "w_gate", None, one)
        expert, weight, counts, balance, offs, place = self.choose(logits, True)
        xs = self.hand_out(n, place, offs)
        a, z_up = self.linear(xs, "w_up", "b_up", offs, B.ACT_GELU, True)
        o = self.linear(a, "w_down", "b_down", offs)
        s = self.dropout(self.together(o, place, weight, offs), h) if train else self.together(o, place, weight, offs, h)
        y = self.linear(s, "w_out", "b_out", one)
        return y, dict(x=x, one=one, h=h, z_in=z_in, n=n, inv=inv, logits=logits, expert=expert, weight=weight, counts=counts, balance=balance, offs=offs, place=place, xs=xs, a=a, z_up=z_up,
                       o=o, s=s)

    def backward(self, clean, y, f):
        """All gradients; the squared error."""
        off = y.float() - clean
        dy = (off * (2.0 / off.numel())).bfloat16()
        n, one, offs, place = len(clean), f["one"], f["offs"], f["place"]
        self.gradients(f["s"], dy, "w_out", "b_out", one)
        ds = self.back(dy, "w_out", one)
        dc = self.dropout(ds, None)
        do, dweight = new(n * K, WIDE), new(n, K, dtype=torch.float32)
        B.combine_rows_backward(BF16, at(dc), WIDE, at(f["o"]), WIDE, at(place), at(f["weight"]), at(offs), EXPERTS, K, n, WIDE, at(do), WIDE, at(dweight), stream())
        self.gradients(f["a"], do, "w_down", "b_down", offs)
        dz = self.back(do, "w_down", offs, None, B.ACT_GELU, f["z_up"])
        self.gradients(f["xs"], dz, "w_up", "b_up", offs)
        dn = self.together(self.back(dz, "w_up", offs), place, None, offs)
        dlogits = new(n, EXPERTS)
        B.route_backward(BF16, at(f["logits"]), EXPERTS, n, EXPERTS, K, True, at(f["expert"]), at(dweight), at(f["counts"]), BALANCE, at(dlogits), EXPERTS, stream())
        self.gradients(f["n"], dlogits, "w_gate", None, one)
        dn = self.back(dlogits, "w_gate", one, dn)
        dh, size = new(n, WIDE), B.rms_norm_backward_bytes(n, WIDE)
        B.rms_norm_backward(BF16, at(dn), WIDE, at(f["h"]), WIDE, at(self.p["gain"]), at(f["inv"]), at(ds), WIDE, n, WIDE, at(dh), WIDE, at(self.g["gain"]), at(new(size, dtype=torch.uint8)),
                            size, stream())
        self.gradients(f["x"], self.through(dh, f["z_in"], "b_in", one, B.ACT_GELU), "w_in", None, one)
        return (off * off).mean()

    def update(self, lr=1e-3):
        self.t += 1
        self.step_on_device += 1
        self.optimizer.step(lr, 0.9, 0.999, 1e-8, self.t, 1, stream())

    def train_step(self, clean, noisy):
        y, f = self.forward(noisy)
        error = self.backward(clean, y, f)
        self.update()
        return error, f["balance"]

    # serving in 8 bits
    def quantized(self, x, precision=BF16):
        """(codes, scales) of a matrix, or of every expert's."""
        cols = x.shape[-1]
        wide = -(-cols // 128) * 128
        q, scale = new(*x.shape[:-1], wide, dtype=torch.uint8), new(*x.shape[:-1], wide // 128, dtype=torch.uint8)
        B.quantize8(precision, at(x), cols, x.numel() // cols, cols, at(q), at(scale), stream())
        return q, scale

    def freeze(self):
        self.w8 = {k: self.quantized(self.p[k], FP32) for k in self.SHAPES if k != "w_gate"}

    def linear8(self, x, name, bias, offs, act=B.ACT_NONE):
        groups, n_out, n_in = self.SHAPES[name]
        y = new(len(x), n_out)
        B.group_linear8_act(*(at(v) for v in self.quantized(x) + self.w8[name]), at(offs), groups, len(x), n_in, n_out, at(self.p[bias]), act, 0, 0, BF16, at(y), n_out, stream())
        return y

    def serve(self, x):
        one = torch.zeros(2, dtype=torch.int32, device="cuda")
        one[1:] = len(x)
        h = self.linear8(x, "w_in", "b_in", one, B.ACT_GELU)
        n, _ = self.norm(h)
        _, weight, _, _, offs, place = self.choose(self.linear(n, "w_gate", None, one), False)
        o = self.linear8(self.linear8(self.hand_out(n, place, offs), "w_up", "b_up", offs, B.ACT_GELU), "w_down", "b_down", offs)
        return self.linear8(self.together(o, place, weight, offs, h), "w_out", "b_out", one)


def main(steps=200, n=1280):
    torch.cuda.set_device(0)
    model, seen = Denoiser(), []
    for k in range(steps):
        seen.append(model.train_step(*batch(n, k)))
    errors, balances = [float(e) for e, _ in seen], [float(b) for _, b in seen]
    clean, noisy = batch(64, 10 ** 6)
    model.freeze()
    exact, served = model.forward(noisy, train=False)[0].float(), model.serve(noisy).float()
    error, noise = float(((served - clean) ** 2).mean()), float(((noisy.float() - clean) ** 2).mean())
    off = float((served - exact).norm() / exact.norm())
    print("squared error: %.4f before training, %.4f after %d steps, %.4f served in 8 bits (of the noisy images: %.4f); balance %.3f, then %.3f; 8-bit outputs differ by %.3f of their norm"
          % (errors[0], errors[-1], steps, error, noise, balances[0], balances[-1], off))
    return errors, balances, error, noise, off


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
