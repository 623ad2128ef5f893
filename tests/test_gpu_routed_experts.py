"""The operators of a layer of experts together (GPU), as the example uses them: it trains and serves, its gradients are those of the same network in 64 bits, and a step captured into a graph and
replayed has the eager step's bits."""
import importlib.util
import os

import numpy as np
import pytest

from tests import experts_ref as R
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("routed_experts", os.path.join(ROOT, "examples", "routed_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs():
    errors, balances, error, noise, off = example().main(8)
    assert len(errors) == 8 and np.all(np.isfinite(errors + balances + [error, noise, off]))


def test_gradients_of_the_whole_step():
    """Every gradient against the same network in 64 bits with the same choices and mask (torch's autograd on the CPU).  The bf16 step rounds what it stores, some two dozen times on the way to the
    first weights, each off by 2^-9 of the norm on average of its size at most: as many independent ones as sqrt(24) * 2^-8, and five times that for the spread of single tensors."""
    torch = U.torch_mod()
    E = example()
    e = E.Denoiser()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    for k in e.BIASES:                                                # (biases of zero would hide theirs)
        e.p[k].copy_(torch.randn(e.p[k].shape, generator=gen, device="cuda") * 0.2)
    n, step = 300, 6
    clean, noisy = E.batch(n, 5)
    e.step_on_device.fill_(step)
    y, f = e.forward(noisy)
    e.backward(clean, y, f)
    torch.cuda.synchronize()
    p = {k: (e.w[k] if k in e.SHAPES else e.p[k]).double().cpu().requires_grad_() for k in e.p}
    expert, counts = f["expert"].cpu().long(), f["counts"].cpu().double()
    keep, scale = R.keep(n, E.WIDE, E.DROP, E.SEED, 0, step)
    keep = torch.from_numpy(keep.astype(np.float64) * scale)

    def gelu(z):
        return z * 0.5 * torch.special.erfc(-z / 2 ** 0.5)

    x = noisy.double().cpu()
    h = gelu(x @ p["w_in"][0].T + p["b_in"][0])
    norm = h / torch.sqrt((h * h).mean(1, keepdim=True) + E.EPS) * p["gain"]
    prob = torch.softmax(norm @ p["w_gate"][0].T, 1)
    chosen = prob.gather(1, expert)
    weight = chosen / chosen.sum(1, keepdim=True)
    parts = []
    for k in range(E.EXPERTS):
        parts.append(gelu(norm @ p["w_up"][k].T + p["b_up"][k]) @ p["w_down"][k].T + p["b_down"][k])
    out = torch.stack(parts, 1).gather(1, expert[:, :, None].expand(-1, -1, E.WIDE))
    s = h + keep * (weight[:, :, None] * out).sum(1)
    got = s @ p["w_out"][0].T + p["b_out"][0]
    balance = E.EXPERTS * (counts[:-1] / counts[:-1].sum() * prob.mean(0)).sum()
    (((got - clean.double().cpu()) ** 2).mean() + E.BALANCE * balance).backward()
    balance, got = float(balance.detach()), got.detach()
    assert abs(float(f["balance"]) - balance) <= 0.01 * balance
    assert float((y.double().cpu() - got).norm() / got.norm()) <= np.sqrt(12) * 2.0 ** -8
    for k in p:
        a, b = e.g[k].double().cpu(), p[k].grad
        assert float((a - b).norm() / b.norm()) <= 5 * np.sqrt(24) * 2.0 ** -8, (k, float((a - b).norm() / b.norm()))


def test_the_step_in_a_graph_and_on_another_stream():
    """Forward and backward captured once, replayed on other batches between eager steps: the same bits as the eager steps every time, each with its own step's mask."""
    torch = U.torch_mod()
    E = example()
    eager, graphed = E.Denoiser(), E.Denoiser()
    batches = [E.batch(500, k) for k in range(4)]
    held = [t.clone() for t in batches[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                     # warm-up outside the capture
        y, f = graphed.forward(held[1])
        graphed.backward(held[0], y, f)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, eager.forward(held[1])[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, f = graphed.forward(held[1])
        graphed.backward(held[0], y, f)
    for clean, noisy in batches:
        held[0].copy_(clean)
        held[1].copy_(noisy)
        graph.replay()
        graphed.update()
        got, g = eager.forward(noisy)
        eager.backward(clean, got, g)
        eager.update()
        torch.cuda.synchronize()
        assert torch.equal(y, got) and torch.equal(f["expert"], g["expert"]) and torch.equal(f["counts"], g["counts"]) and torch.equal(f["balance"], g["balance"])
        for k in eager.p:
            assert torch.equal(eager.g[k], graphed.g[k]) and torch.equal(eager.p[k], graphed.p[k]), k


def test_labels_of_a_batch_sorted_on_the_device():
    """What a program with labels does in place of the host's sort: the rows of a mixed batch through their experts and back into the batch's order.  Whole numbers."""
    from paper_2102_10485_amd import binding as B
    torch = U.torch_mod()
    labels, n, n_in, n_out = 9, 3000, 72, 40
    rng = np.random.default_rng(8)
    lab = rng.integers(-1, labels, n).astype(np.int32)                # (some without a label: zeros)
    lab[lab == 4] = 5
    x, w = rng.integers(-2, 3, (n, n_in)).astype(np.float32), rng.integers(-2, 3, (labels, n_out, n_in)).astype(np.float32)
    tl, tx, tw = torch.from_numpy(lab).cuda(), torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    offs, place, xs, ys, y = torch.empty(labels + 1, dtype=torch.int32, device="cuda"), torch.empty_like(tl), torch.empty_like(tx), torch.empty((n, n_out), device="cuda"), torch.empty((n, n_out), device="cuda")
    size = B.sort_by_label_bytes(n, labels)
    work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    B.sort_by_label(tl.data_ptr(), n, labels, offs.data_ptr(), 0, place.data_ptr(), work.data_ptr(), size)
    B.gather_rows(B.FP32, tx.data_ptr(), n_in, place.data_ptr(), offs.data_ptr(), labels, 1, n, n_in, xs.data_ptr(), n_in)
    B.group_linear_act(B.FP32, xs.data_ptr(), n_in, tw.data_ptr(), offs.data_ptr(), labels, n, n_in, n_out, 0, B.ACT_RELU, 0, 0, 0, 0, ys.data_ptr(), n_out)
    B.combine_rows(B.FP32, ys.data_ptr(), n_out, place.data_ptr(), 0, offs.data_ptr(), labels, 1, 0, 0, n, n_out, y.data_ptr(), n_out)
    want = np.maximum(np.einsum("ni,noi->no", x, w[lab]), 0) * (lab >= 0)[:, None]
    assert np.array_equal(y.cpu().numpy(), want)
