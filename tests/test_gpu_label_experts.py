"""The operators together (GPU): the example's training and serving, the same step replayed from a HIP graph, and another stream."""
import importlib.util
import os

import numpy as np
import pytest

from tests import gpu_util as U

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("label_experts", os.path.join(ROOT, "examples", "label_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_learns_and_serves():
    """Denoising: the error falls below the noise's own (0.25) by far; 8-bit values are off by at most 2^-4 each, independently, on both sides of three products."""
    losses, error, noise, off = example().main(60)
    assert np.all(np.isfinite(losses)) and losses[-1] < 0.5 * losses[0]
    assert losses[-1] < 0.2 * noise and error < 0.25 * noise
    assert off < 3 * np.sqrt(2) * 2.0 ** -4


def test_gradients_of_the_whole_step():
    """Every gradient against the same network in 64 bits, differentiated by hand in another form (torch's autograd on the CPU).  The bf16 step rounds what it stores, a dozen
    times on the way to the first weights: 12 * 2^-9 of the norm, and as much again."""
    torch = U.torch_mod()
    E = example()
    e = E.Experts()
    clean, noisy, offs = E.batch(200, 5)
    p = {k: e.w[k].double().cpu().requires_grad_() if k.startswith("w") else e.p[k].double().cpu().requires_grad_() for k in e.p}
    e.train_step(clean, noisy, offs)
    o = offs.cpu().tolist()

    def linear(x, w):
        return torch.cat([x[o[g]:o[g + 1]] @ w[g].T for g in range(E.LABELS)])

    def norm(x, gain):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + E.EPS) * gain

    h = linear(noisy.double().cpu(), p["w_in"])
    s = h + linear(norm(h, p["gain_mid"]), p["w_mid"])
    y = linear(norm(s, p["gain_out"]), p["w_out"])
    ((y - clean.double().cpu()) ** 2).mean().backward()
    for k in p:
        got, want = e.g[k].double().cpu(), p[k].grad
        assert float((got - want).norm() / want.norm()) <= 24 * 2.0 ** -9, k


def test_the_step_in_a_graph_and_on_another_stream():
    """Captured once and replayed with other batches between eager work: the same bits as the eager step every time."""
    torch = U.torch_mod()
    E = example()
    eager, graphed = E.Experts(), E.Experts()
    batches = [E.batch(300, k) for k in range(4)]
    held = [t.clone() for t in batches[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                     # warm-up outside the capture, then back to the start
        y = graphed.forward(held[1], held[2])[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, eager.forward(held[1], held[2])[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, (h, n1, inv1, s, n2, inv2) = graphed.forward(held[1], held[2])
        dy = ((y.float() - held[0]) * (2.0 / y.numel())).bfloat16()
        ds = graphed.norm_backward(graphed.linear_backward(n2, dy, "w_out", held[2]), s, inv2, None, "gain_out")
        dh = graphed.norm_backward(graphed.linear_backward(n1, ds, "w_mid", held[2]), h, inv1, ds, "gain_mid")
        graphed.linear_backward(held[1], dh, "w_in", held[2], want_dx=False)
    for clean, noisy, offs in batches:
        for t, v in zip(held, (clean, noisy, offs)):
            t.copy_(v)
        graph.replay()
        graphed.t += 1
        graphed.optimizer.step(1e-3, 0.9, 0.999, 1e-8, graphed.t, 1, E.stream())
        eager.train_step(clean, noisy, offs)
        torch.cuda.synchronize()
        for k in eager.p:
            assert torch.equal(eager.g[k], graphed.g[k]) and torch.equal(eager.p[k], graphed.p[k]), k
    for a, b in zip(eager.moments + eager.scales, graphed.moments + graphed.scales):
        assert torch.equal(a, b)


def test_rows_sorted_by_a_training_steps_routing():
    """The routing that a DC-CGAN context reports, on the host, sorts other rows of the same batch for the products: its offsets are copied to the device as they are.  Whole numbers."""
    from paper_2102_10485_amd import binding as B
    from paper_2102_10485_amd import synth
    torch = U.torch_mod()
    labels, n, n_in, n_out = 9, 300, 72, 40
    rng = np.random.default_rng(8)
    lab = rng.integers(0, labels, n).astype(np.int32)
    lab[lab == 4] = 5                                                 # a label without rows
    spec = synth.SPECS["tiny0"]
    gan = B.Gan(B.make_config(spec, labels, labels, n, B.BF16), torch.cuda.current_stream().cuda_stream)
    z, image = rng.normal(size=(n, spec["z_dim"])), np.tanh(rng.normal(size=(n, spec["img_c"], spec["img_hw"], spec["img_hw"])))
    dl, dz, dimage = torch.from_numpy(lab).cuda(), torch.from_numpy(z.astype(np.float32)).cuda(), torch.from_numpy(image.astype(np.float32)).cuda()
    gan.train_step(dl.data_ptr(), dz.data_ptr(), dimage.data_ptr(), n)
    perm, offs = gan.get_routing(n)
    gan.close()
    x, w = rng.integers(-2, 3, (n, n_in)).astype(np.float32), rng.integers(-2, 3, (labels, n_out, n_in)).astype(np.float32)
    tx, tw, to = torch.from_numpy(x[perm]).cuda().bfloat16(), torch.from_numpy(w).cuda().bfloat16(), torch.from_numpy(offs).cuda()
    y = torch.empty((n, n_out), dtype=torch.bfloat16, device="cuda")
    B.group_linear(B.BF16, tx.data_ptr(), n_in, tw.data_ptr(), to.data_ptr(), labels, n, n_in, n_out, y.data_ptr(), n_out)
    got = np.empty((n, n_out), np.float32)
    got[perm] = y.float().cpu().numpy()
    assert np.array_equal(got, U.round_to(np.einsum("ni,noi->no", x, w[lab]), True))
