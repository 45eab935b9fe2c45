"""4-bit layers and AdamW together, as a training step has them: weights, inputs and gradients rounded to 4 bits along the
axis that each product sums over, the forward pass, both backward products, the update.  Every step is compared with the plain
definition, which is fed the GPU's own inputs of that step; the gradients also with differences of the GPU's own outputs."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def G():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gpu_util
    return gpu_util


@pytest.fixture(scope="module")
def bnn():
    import paper_1706_09453_amd as b
    return b


def f32(*shape):
    return torch.full(shape, float("nan"), dtype=torch.float32, device=DEV)


def matrix(bnn, R, K):
    return torch.empty(bnn.bnn_mx4_bytes(R, K), dtype=torch.uint8, device=DEV)


class Net:
    """440-like small network: 4-bit Sigmoid layers and a 4-bit Softmax layer, trained by AdamW with 8- or 32-bit states."""

    def __init__(self, G, bnn, dims, M, bits, seed):
        rng = np.random.default_rng(seed)
        self.G, self.bnn, self.dims, self.M, self.bits, self.L = G, bnn, dims, M, bits, len(dims) - 1
        self.W = [G.to_dev((rng.uniform(-1, 1, (n, k)) * np.sqrt(3.0 / k)).astype(np.float32)) for k, n in zip(dims, dims[1:])]
        self.b = [G.to_dev((rng.standard_normal(n) * 0.1).astype(np.float32)) for n in dims[1:]]
        self.X = G.to_dev(rng.standard_normal((M, dims[0])).astype(np.float32))
        self.labels = G.to_dev(rng.integers(0, dims[-1], M).astype(np.int32))
        shapes = list(zip(dims, dims[1:]))
        self.Wq, self.WqT = [matrix(bnn, n, k) for k, n in shapes], [matrix(bnn, k, n) for k, n in shapes]
        self.hq, self.hqT = [matrix(bnn, M, k) for k, _ in shapes], [matrix(bnn, k, M) for k, _ in shapes]
        self.gq, self.gqT = [matrix(bnn, M, n) for _, n in shapes], [matrix(bnn, n, M) for _, n in shapes]
        self.h = [self.X] + [f32(M, n) for _, n in shapes]
        self.g = [f32(M, n) for _, n in shapes]
        self.gh = [None] + [f32(M, k) for k, _ in shapes[1:]]
        self.gw, self.gb = [f32(n, k) for k, n in shapes], [f32(n) for _, n in shapes]
        self.step = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.state, descs = [], []
        for w, g in [(w, g) for pair in zip(zip(self.W, self.gw), zip(self.b, self.gb)) for w, g in pair]:
            n = w.numel()
            kind = torch.float32 if bits == 32 else torch.uint8
            s = {"m": torch.zeros(n, dtype=kind, device=DEV), "v": torch.zeros(n, dtype=kind, device=DEV)}
            if bits == 8:
                s |= {k: torch.zeros((n + 31) // 32, dtype=torch.uint8, device=DEV) for k in ("m_scale", "v_scale")}
            self.state.append(s)
            descs.append({"w": w.data_ptr(), "g": g.data_ptr(), "count": n, "clip": w.dim() == 2} | {k: t.data_ptr() for k, t in s.items()})
        self.list = bnn.make_adamw_array(descs)

    def seed(self, l, step):
        return l * (1 << 40) + step

    def quantize(self, X, Q, QT, rounding, seed, st, on_device=False):
        R, C = X.shape
        if on_device:   # the seed, and the step's number there
            self.bnn.bnn_quantize_mx4_step(X.data_ptr(), R, C, seed, self.step.data_ptr(), Q.data_ptr(), QT.data_ptr(), st)
            return
        self.bnn.bnn_quantize_mx4(X.data_ptr(), R, C, rounding, seed, Q.data_ptr(), QT.data_ptr(), st)

    def forward(self, st):
        b = self.bnn
        for l in range(self.L):
            n, k = self.W[l].shape
            self.quantize(self.W[l], self.Wq[l], self.WqT[l], b.BNN_ROUND_NEAREST, 0, st)
            self.quantize(self.h[l], self.hq[l], self.hqT[l], b.BNN_ROUND_NEAREST, 0, st)
            act = b.BNN_ACT_SIGMOID if l + 1 < self.L else b.BNN_ACT_LOGSOFTMAX
            b.bnn_layer_mx4(self.hq[l].data_ptr(), self.Wq[l].data_ptr(), self.b[l].data_ptr(), self.M, k, n, act, 32, self.h[l + 1].data_ptr(), st)

    def backward(self, step, st, on_device=False):
        b, M = self.bnn, self.M
        b.bnn_softmax_xent_grad(self.h[-1].data_ptr(), self.labels.data_ptr(), M, self.dims[-1], self.g[-1].data_ptr(), st)
        for l in range(self.L - 1, -1, -1):
            n, k = self.W[l].shape
            if l + 1 < self.L:
                b.bnn_sigmoid_grad(self.gh[l + 1].data_ptr(), self.h[l + 1].data_ptr(), M * n, self.g[l].data_ptr(), st)
            self.quantize(self.g[l], self.gq[l], self.gqT[l], b.BNN_ROUND_STOCHASTIC, self.seed(l, step), st, on_device)
            b.bnn_layer_mx4(self.gqT[l].data_ptr(), self.hqT[l].data_ptr(), 0, n, M, k, b.BNN_ACT_LINEAR, 32, self.gw[l].data_ptr(), st)
            b.bnn_bias_grad(self.g[l].data_ptr(), M, n, self.gb[l].data_ptr(), st)
            if l > 0:
                b.bnn_layer_mx4(self.gq[l].data_ptr(), self.WqT[l].data_ptr(), 0, M, n, k, b.BNN_ACT_LINEAR, 32, self.gh[l].data_ptr(), st)

    HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.01)

    def update(self, step, st, on_device=False):
        p = self.bnn.bnn_adamw_params(**self.HYPER, step=0 if on_device else step, state_bits=self.bits, seed=7 if on_device else 7 + step, step_at=self.step.data_ptr() if on_device else 0)
        self.bnn.bnn_update_adamw(self.list, 2 * self.L, p, st)

    def tensors(self):
        return self.h[1:] + self.g + self.gw + self.gb + self.W + self.b + [t for s in self.state for t in s.values()]


def product_is(got, x, w, bias=0.0):
    """x w^T + bias in fp32 sums of any order (test_gpu_mx4.py says where the bound comes from)."""
    h = x @ w.T + bias
    off = x.shape[1] * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + 2.0 ** -23 * (np.abs(h) + np.abs(bias))
    assert (np.abs(got - h) <= off).all()


@pytest.mark.parametrize("bits,M,dims", [(32, 70, (40, 96, 33)), (8, 200, (130, 257, 64, 50)), (8, 1, (33, 20, 5))])
def test_steps_of_training(G, bnn, bits, M, dims):
    net = Net(G, bnn, dims, M, bits, M)
    st = G.stream()
    for step in (1, 2, 3):
        net.forward(st)
        host = lambda t: t.cpu().numpy()   # noqa: E731
        for l in range(net.L):
            n, k = net.W[l].shape
            hq, wq = mx.unpack(mx.quantized(host(net.h[l])), M, k), mx.unpack(mx.quantized(host(net.W[l])), n, k)
            z = hq @ wq.T + host(net.b[l])
            off = k * 2.0 ** -24 * (np.abs(hq) @ np.abs(wq).T) + 2.0 ** -23 * (np.abs(z) + np.abs(host(net.b[l])))
            got = host(net.h[l + 1])
            if l + 1 < net.L:
                assert (np.abs(got - 1 / (1 + np.exp(-z))) <= off / 4 + 2.0 ** -24).all()
            else:
                top = z.max(1, keepdims=True)
                want = z - top - np.log(np.exp(z - top).sum(1, keepdims=True))
                assert (np.abs(got - want) <= off + off.max(1, keepdims=True) + 2.0 ** -20 * (1 + np.abs(z).max(1, keepdims=True) + np.abs(want))).all()
        net.backward(step, st)
        for l in range(net.L - 1, -1, -1):
            n, k = net.W[l].shape
            g = host(net.g[l])
            rows = mx.unpack(mx.quantized(g, mx.STOCHASTIC, net.seed(l, step)), M, n)
            columns = mx.unpack(mx.quantized(g, mx.STOCHASTIC, net.seed(l, step), columns=True), n, M)
            product_is(host(net.gw[l]), columns, mx.unpack(mx.quantized(host(net.h[l]), columns=True), k, M))
            if l > 0:
                product_is(host(net.gh[l]), rows, mx.unpack(mx.quantized(host(net.W[l]), columns=True), k, n))
        before = [{k: host(t).copy() for k, t in s.items()} | {"w": host(w).reshape(-1).copy(), "g": host(g).reshape(-1)}
                  for s, w, g in zip(net.state, [t for p in zip(net.W, net.b) for t in p], [t for p in zip(net.gw, net.gb) for t in p])]
        net.update(step, st)
        for i, (a, w, s) in enumerate(zip(before, [t for p in zip(net.W, net.b) for t in p], net.state)):
            kw = dict(net.HYPER, clip=i % 2 == 0)
            if bits == 32:
                want_w, m, v, _ = mx.adamw(a["w"], a["g"], a["m"], a["v"], step, **kw)
                want = {"m": m, "v": v}
            else:
                want_w, m, ms, v, vs = mx.adamw8(a["w"], a["g"], a["m"].view(np.int8), a["m_scale"], a["v"], a["v_scale"], step, 7 + step, i, **kw)
                want = {"m": m.view(np.uint8), "m_scale": ms, "v": v, "v_scale": vs}
            assert np.array_equal(host(w).reshape(-1), want_w), i
            for k in want:
                assert np.array_equal(host(s[k]), want[k]), (i, k)


def test_a_captured_step_is_the_eager_one(G, bnn):
    """The whole step in a graph, replayed with the step's number on the device, against the same network stepped eagerly."""
    for bits in (8, 32):
        a, b = (Net(G, bnn, (100, 160, 70), 96, bits, 5) for _ in range(2))
        st = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            a.forward(st.cuda_stream)
            a.backward(0, st.cuda_stream, on_device=True)
            a.update(0, st.cuda_stream, on_device=True)
        for step in range(1, 5):
            a.step.fill_(step)
            a.X.copy_(torch.randn(a.X.shape, device=DEV))
            b.X.copy_(a.X)
            torch.cuda.synchronize()
            graph.replay()
            b.forward(G.stream())
            b.backward(step, G.stream())
            b.update(step, G.stream())
            torch.cuda.synchronize()
            for x, y in zip(a.tensors(), b.tensors()):
                assert torch.equal(x, y) and (x.dtype != torch.float32 or torch.isfinite(x).all()), (bits, step)


def test_gradients_against_differences(G, bnn):
    """With numbers that 4 bits hold exactly, along rows and along columns, the backward products are the gradient of the layer: of
    loss = sum c * (X W^T), whose differences the layer itself gives for inputs and weights that go one up and one down."""
    M, K, N = 33, 70, 40
    rng = np.random.default_rng(0)
    X, W, c = (rng.integers(-1, 2, s).astype(np.float32) for s in ((M, K), (N, K), (M, N)))
    st = G.stream()

    def forms(A):
        q, t = matrix(bnn, *A.shape), matrix(bnn, *A.shape[::-1])
        d = G.to_dev(A)
        bnn.bnn_quantize_mx4(d.data_ptr(), *A.shape, 0, 0, q.data_ptr(), t.data_ptr(), st)
        return q, t

    def product(x, w, m, k, n):
        y = f32(m, n)
        bnn.bnn_layer_mx4(x.data_ptr(), w.data_ptr(), 0, m, k, n, bnn.BNN_ACT_LINEAR, 32, y.data_ptr(), st)
        return y.cpu().numpy().astype(np.float64)

    def loss(X, W):
        return (c * product(forms(X)[0], forms(W)[0], M, K, N)).sum()

    gx = product(forms(c)[0], forms(W)[1], M, N, K)
    gw = product(forms(c)[1], forms(X)[1], N, M, K)
    for _ in range(12):
        m, n, k = rng.integers(M), rng.integers(N), rng.integers(K)
        for A, grad, at in ((X, gx, (m, k)), (W, gw, (n, k))):
            up, down = A.copy(), A.copy()
            up[at] += 1
            down[at] -= 1
            d = (loss(up, W) - loss(down, W)) / 2 if A is X else (loss(X, up) - loss(X, down)) / 2
            assert d == grad[at]
