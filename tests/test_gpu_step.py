"""Layer norm, the gated block, the linear layer and AdamW together, as a training step uses them:
y = linear(gated(norm(x))) + x, its gradients and the weights' step. The parts against plain references of their own
inputs; the whole on other streams, captured and replayed, and two graphs at once, bit for bit."""
import numpy as np
import pytest
import torch

import narrow_ref
import step_ref as ref
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


class Block:
    """float32 weights, bfloat16 copies, moments in 8 bits or float32; everything of a step in `out`."""

    def __init__(self, hf, width, hidden, fmt, seed=1):
        self.hf = hf
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        w = [torch.ones(width), torch.zeros(width), r(hidden, width) / width ** 0.5, r(hidden, width) / width ** 0.5,
             r(width, hidden) / hidden ** 0.5, torch.zeros(width)]
        self.weights = [t.cuda() for t in w]
        # the norm's weight and bias are read as they are, the products' in 16 bits
        self.copies = [None, None] + [t.bfloat16() for t in self.weights[2:]]
        self.state = hf.adamw_state(self.weights, fmt)

    def forward(self, x):
        hf, (nw, nb, *_), (_, _, gate, up, down, bias) = self.hf, self.weights, self.copies
        n, kept = hf.layer_norm(x, nw, nb, save=True)
        h, saved = hf.gated_forward(n, gate, up, ckpt=(4, 3))
        return hf.linear(h, down, bias, residual=x), (n, kept, h, saved)

    def backward(self, x, dy, kept):
        hf, nw, (_, _, gate, up, down, _) = self.hf, self.weights[0], self.copies
        n, norm, h, saved = kept
        dh, ddown, dbias = hf.linear_backward(dy, h, down)
        dn, dgate, dup = hf.gated_backward(dh, saved, gate, up)
        dx, dnw, dnb = hf.layer_norm_backward(dn, x, norm, nw, add=dy)
        return dx, [t.bfloat16() for t in (dnw, dnb)] + [dgate, dup, ddown, dbias], (dh, dn)

    def step(self, x, dy, number, **kw):
        y, kept = self.forward(x)
        dx, grads, _ = self.backward(x, dy, kept)
        self.hf.adamw(self.weights, grads, self.state, number, copies=self.copies, seed=7, **kw)
        return y, dx

    def all(self):
        s = self.state
        return self.weights + self.copies[2:] + ([s.m, s.v] if s.fmt is None else [*s.m, *s.v])


def _data(T, width, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, width, generator=g).bfloat16().cuda() for _ in range(2)]


def _same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("T,width,hidden", [(1, 64, 96), (33, 100, 171), (200, 264, 520)])
def test_the_parts_of_a_step(T, width, hidden):
    """Each operator's results from what the one before it gave; tolerances as in the operators' own tests, with
    a step of bfloat16 (2^-7) where several of its halves meet."""
    hf = need_gpu()
    say("step", T, width, hidden)
    block = Block(hf, width, hidden, (4, 3))
    x, dy = _data(T, width, 2)
    d = lambda t: t.double().cpu().numpy()  # noqa: E731
    y, kept = block.forward(x)
    n, norm, h, saved = kept
    nw, nb = (d(t) for t in block.weights[:2])
    gate, up, down, bias = (d(t) for t in block.copies[2:])
    half = ref.HALF["bf16"]
    want, mean, rstd, xh = ref.layer_norm(d(x), nw, nb, 1e-5)
    assert (np.abs(d(n) - want) <= half * np.abs(want) + 2.0 ** -18 * (1 + np.abs(want))).all()
    want = d(h) @ down.T + bias + d(x)
    slack = (hidden + 2) * 2.0 ** -23 * (np.abs(d(h)) @ np.abs(down).T + np.abs(want))
    assert (np.abs(d(y) - want) <= half * np.abs(want) + slack).all()
    dx, grads, (dh, dn) = block.backward(x, dy, kept)
    for got, want, size in ((dh, d(dy) @ down, np.abs(d(dy)) @ np.abs(down)),
                            (grads[4], d(dy).T @ d(h), np.abs(d(dy)).T @ np.abs(d(h))),
                            (grads[5], d(dy).sum(0), np.abs(d(dy)).sum(0))):
        assert (np.abs(d(got) - want) <= half * np.abs(want) + (T + hidden) * 2.0 ** -23 * size).all()
    # the gated block's gradients from its blocks' values
    values = [narrow_ref.unpack(c.cpu().numpy().astype(np.int64), np.exp2(s.cpu().double().numpy() - 127), (4, 3))
              for c, s in (saved.x, saved.gate, saved.up)]
    a, da = narrow_ref.act(values[1], 0)
    dg, du = d(dh) * values[2] * da, d(dh) * a
    size = np.abs(dg) @ np.abs(gate) + np.abs(du) @ np.abs(up)
    assert (np.abs(d(dn) - dg @ gate - du @ up) <= half * np.abs(d(dn)) + 1.01 * half * size).all()
    want, ww, wb = ref.layer_norm_grad(d(dn), xh, rstd, nw, d(dy))
    # (of the sum's two terms: the larger's float32 error)
    assert (np.abs(d(dx) - want) <= half * np.abs(want) + 2.0 ** -17 * (rstd * np.abs(d(dn)).max() + np.abs(d(dy)))).all()
    before = [d(t) for t in block.weights]
    hf.adamw(block.weights, grads, block.state, 1, copies=block.copies, lr=1e-2, weight_decay=0.0)
    for w, b, g in zip(block.weights, before, grads):
        # a first step is lr in the direction of the gradient's sign, where it is far above eps
        moved, g = d(w) - b, d(g)
        far = np.abs(g) > 1e-4
        assert (np.abs(moved + 1e-2 * np.sign(g))[far] <= 1e-2 * 2e-4 + 2.0 ** -23 * np.abs(b)[far]).all()
    assert _same(block.copies[2:], [w.bfloat16() for w in block.weights[2:]])


@pytest.mark.parametrize("fmt", [None, (4, 3)])
def test_on_other_streams(fmt):
    hf = need_gpu()
    data = [_data(77, 128, s) for s in range(3)]
    a, b = (Block(hf, 128, 256, fmt) for _ in range(2))
    want = [a.step(*d, i + 1) for i, d in enumerate(data)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i, (s, d) in enumerate(zip(streams, data)):
        s.wait_stream(streams[i - 1] if i else torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(b.step(*d, i + 1))
    torch.cuda.synchronize()
    assert all(_same(p, q) for p, q in zip(want, got)) and _same(a.all(), b.all())


@pytest.mark.parametrize("fmt", [None, (5, 2)])
@pytest.mark.parametrize("T", [1, 77])
def test_captured_and_replayed(fmt, T):
    """A whole step in a graph, with the step's number and the rate on the device, replayed with other inputs
    between eager steps of another block."""
    hf = need_gpu()
    data = [_data(T, 128, s) for s in range(5)]
    a, b = (Block(hf, 128, 256, fmt) for _ in range(2))
    number = torch.tensor([1], device="cuda")
    rate = torch.tensor([1e-2], device="cuda")
    count = torch.tensor([1], device="cuda")      # the eager one's
    x, dy = (t.clone() for t in data[0])

    def eager(block, d):
        out = block.step(*d, count, lr=rate)
        count.add_(1)
        return out

    # (warm on another stream, on a block that is thrown away)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Block(hf, 128, 256, fmt).step(x, dy, number, lr=rate)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = b.step(x, dy, number, lr=rate)
        number.add_(1)
    other = Block(hf, 128, 256, fmt, seed=2)
    for i, d in enumerate(data):
        want = eager(a, d)
        x.copy_(d[0])
        dy.copy_(d[1])
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        other.step(*d, i + 1)
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and _same(a.all(), b.all()), i
        rate.mul_(0.5)


def test_two_graphs_at_once():
    """Two captured passes, replayed on two streams at the same time, have workspaces of their own."""
    hf = need_gpu()
    x, dy = _data(300, 520, 3)
    g = torch.Generator().manual_seed(4)
    w = [(torch.randn(264, 520, generator=g) / 20).bfloat16().cuda() for _ in range(2)]
    gy = torch.randn(300, 264, generator=g).bfloat16().cuda()

    def run(i):
        y, z = hf.linear(x, w[i], None, hf.GATE_SILU, save=True)
        n, kept = hf.layer_norm(x, save=True)
        return [y, *hf.linear_backward(gy, x, w[i], z, hf.GATE_SILU), n, *hf.layer_norm_backward(dy, x, kept)]

    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(run(i))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for t in [t for o in outs for t in o]:
            t.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(outs, want))


def test_a_lost_gradient_is_told():
    hf = need_gpu()
    x, dy = _data(5, 64, 5)
    w = torch.ones(64, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    with pytest.warns(UserWarning, match="no gradient"):
        y = hf.linear(x, w)
    assert not y.requires_grad
    with pytest.warns(UserWarning, match="no gradient"):
        hf.layer_norm(x.clone().requires_grad_())
    with torch.no_grad():
        assert torch.equal(hf.linear(x, w), y)


def test_8_bit_states_train_as_float32_ones_do():
    """A thousand steps on the function sum (w - w0)^2 / 2 with noise on its gradient: the mean distance that the
    8-bit states leave is that of the float32 ones within a factor (states that stop moving leave a multiple)."""
    hf = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(6)
    goal = torch.randn(8192, generator=g, device="cuda")
    left = []
    for fmt in (None, (4, 3)):
        noise = torch.Generator(device="cuda").manual_seed(7)
        w = torch.zeros(8192, device="cuda")
        s = hf.adamw_state([w], fmt)
        for step in range(1, 1001):
            grad = (w - goal) + 0.5 * torch.randn(8192, generator=noise, device="cuda")
            hf.adamw([w], [grad], s, step, lr=1e-2, weight_decay=0.0, seed=3)
        left.append((w - goal).abs().mean().item())
        v = s.v if fmt is None else ref.decode(s.v[0].cpu().numpy(), s.v[1].cpu().numpy(), fmt) ** 2
        left.append(float(v.mean()))
    # v of either: the same gradients but for the weights' own way; its rounding's variance is an eighth of v's
    # square a value, over 8192 of them 0.4 % of the mean
    assert abs(left[3] / left[1] - 1) < 0.05
    assert left[2] < 2 * left[0]


def test_columns_of_one_matrix():
    """Inputs and results beside each other in wider rows; what would overlap is refused."""
    hf = need_gpu()
    g = torch.Generator().manual_seed(3)
    for T in (1, 5, 300):
        both = torch.randn(T, 264, generator=g).bfloat16().cuda()
        w = torch.randn(132, 132, generator=g).bfloat16().cuda()
        x, y = both[:, :132], both[:, 132:]
        want = hf.layer_norm(x.clone()), hf.linear(x.clone(), w)
        assert torch.equal(hf.layer_norm(x, out=y), want[0])
        assert torch.equal(hf.linear(x, w, out=y), want[1])
        assert torch.equal(hf.linear(y, w, out=x), hf.linear(want[1], w))
        for out in (x, both[:, 1:133]):
            with pytest.raises(hf.HobflopsError):
                hf.linear(x, w, out=out)
        with pytest.raises(hf.HobflopsError):
            hf.layer_norm(x, out=both[:, 131:263])


def test_results_of_more_than_the_caches():
    """Results from 64 MiB on are stored in another way: the same values as of parts of the rows."""
    hf = need_gpu()
    say("results past the caches")
    g = torch.Generator(device="cuda").manual_seed(4)
    rows, cols = 8200, 4103
    x = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    w = torch.randn(cols, 72, generator=g, device="cuda").bfloat16()
    codes = hf.block_pack(x, (4, 3))
    parts = [slice(0, 4100), slice(4100, rows)]
    y, saved = hf.layer_norm(x, save=True)
    dx = hf.layer_norm_backward(x, y, saved, add=x)[0]
    up = hf.block_unpack(*codes, cols, (4, 3), dtype=torch.bfloat16)
    out, z = hf.linear(y[:, :72].contiguous(), w, None, hf.GATE_RELU, residual=x, save=True)
    for p in parts:
        assert torch.equal(y[p], hf.layer_norm(x[p]))
        assert torch.equal(dx[p], hf.layer_norm_backward(x[p], y[p], hf.NormSaved(saved.mean[p], saved.rstd[p]), add=x[p])[0])
        assert torch.equal(up[p], hf.block_unpack(codes[0][p], codes[1][p], cols, (4, 3), dtype=torch.bfloat16))
        some = hf.linear(y[p, :72].contiguous(), w, None, hf.GATE_RELU, residual=x[p], save=True)
        assert torch.equal(out[p], some[0]) and torch.equal(z[p], some[1])
