"""GPU parity of the 4-bit layers (bnn_quantize_mx4, bnn_dequantize_mx4, bnn_layer_mx4, bnn_layer_mx4_realx) with the plain
definitions in oracle/mx_oracle.py.

Codes and scale bytes are compared byte for byte.  Sums: a sum of K products in fp32, in any order, is off by at most
K 2^-24 sum_k |x_k w_k| (K - 1 additions, each rounded by half a step of a partial sum that is no larger than the sum of
magnitudes), the bias by one more rounding.  Where all partial sums are multiples of a power of two below 2^24 of them,
they are exact in any order, and the outputs are compared bit for bit."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu

GUARD = 64


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


class Buffer:
    """nbytes of device memory, filled with a pattern, between guards that have to keep theirs; offset: bytes past 256-byte alignment."""

    def __init__(self, nbytes, offset=0):
        self.n, self.from_ = nbytes, 256 + offset
        self.t = torch.full((self.from_ + nbytes + GUARD,), 0xA5, dtype=torch.uint8, device="cuda:0")
        self.ptr = self.t.data_ptr() + self.from_
        assert self.t.data_ptr() % 256 == 0

    def put(self, a):
        self.t[self.from_:self.from_ + self.n] = torch.from_numpy(np.ascontiguousarray(a).reshape(-1).view(np.uint8)).to("cuda:0")
        return self

    def get(self, dtype=np.uint8):
        a = self.t.cpu().numpy()
        assert (a[:self.from_] == 0xA5).all() and (a[self.from_ + self.n:] == 0xA5).all(), "written outside the buffer"
        return a[self.from_:self.from_ + self.n].copy().view(dtype)


def quantize(G, bnn, X, rounding=0, seed=0, rows=True, columns=False, offset=0):
    R, C = X.shape
    x = Buffer(X.nbytes, offset).put(X)
    q = Buffer(bnn.bnn_mx4_bytes(R, C)) if rows else None
    t = Buffer(bnn.bnn_mx4_bytes(C, R)) if columns else None
    bnn.bnn_quantize_mx4(x.ptr, R, C, rounding, seed, q.ptr if q else 0, t.ptr if t else 0, G.stream())
    return q, t


SPECIAL = np.array([0.0, -0.0, 6.0, -6.0, 5.0, -5.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 0.2499999, 0.2500001, 1e-30, -1e-30, 1.2e-38, -5e-39, 1e-45,
                    3.4e38, -3.4e38, 1.0, 2.0, 3.0, 4.0, 0.5, 1.5, -0.25], np.float32)


def matrix(R, C, seed, special=False):
    rng = np.random.default_rng(seed)
    X = (rng.standard_normal((R, C)) * np.exp(3 * rng.standard_normal((R, 1)))).astype(np.float32)
    X[rng.random((R, C)) < 0.1] = 0.0
    X[::5] = 0.0
    if special:   # blocks in which single numbers decide: ties, very small and very large ones, Inf and NaN
        for i in range(max(1, R * C // 40)):
            X[rng.integers(R), rng.integers(C)] = SPECIAL[rng.integers(SPECIAL.size)]
        X[rng.integers(R), rng.integers(C)] = np.nan
        X[rng.integers(R), rng.integers(C)] = np.inf
        X[rng.integers(R), rng.integers(C)] = -np.inf
    return X


SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (7, 127), (1, 128), (5, 129), (33, 40), (64, 440), (128, 128), (130, 259), (257, 130), (1000, 36), (31, 2048),
         (1, 5000), (3000, 1)]


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("R,C", SIZES)
def test_quantize_both_ways(G, bnn, R, C, rounding):
    X = matrix(R, C, R * 7919 + C, special=True)
    q, t = quantize(G, bnn, X, rounding, 0x123456789ABCDEF0 + R, True, True)
    want_q, want_t = mx.quantized(X, rounding, 0x123456789ABCDEF0 + R), mx.quantized(X, rounding, 0x123456789ABCDEF0 + R, True)
    got_q, got_t = q.get(), t.get()
    C4 = (C + 127) // 128
    used = R * C4 * 64
    assert np.array_equal(got_q[:used], want_q[:used]) and np.array_equal(got_q[(used + 255) // 256 * 256:], want_q[(used + 255) // 256 * 256:])
    used = C * ((R + 127) // 128) * 64
    assert np.array_equal(got_t[:used], want_t[:used]) and np.array_equal(got_t[(used + 255) // 256 * 256:], want_t[(used + 255) // 256 * 256:])
    # each form by itself is the same
    for rows in (True, False):
        one = [b for b in quantize(G, bnn, X, rounding, 0x123456789ABCDEF0 + R, rows, not rows) if b][0]
        both = got_q if rows else got_t
        n = (R * C4 if rows else C * ((R + 127) // 128)) * 64
        got = one.get()
        assert np.array_equal(got[:n], both[:n]) and np.array_equal(got[(n + 255) // 256 * 256:], both[(n + 255) // 256 * 256:])


@pytest.mark.parametrize("offset", [4, 8, 12])
def test_quantize_unaligned_input(G, bnn, offset):
    X = matrix(67, 260, offset)
    q, t = quantize(G, bnn, X, 0, 0, True, True, offset)
    n = 67 * 3 * 64
    assert np.array_equal(q.get()[:n], mx.quantized(X)[:n]) and np.array_equal(t.get()[:260 * 64], mx.quantized(X, columns=True)[:260 * 64])


def test_quantize_scales_from_the_smallest_to_the_largest(G, bnn):
    """Every scale byte, with numbers at, just below and just above the borders between them."""
    tops = np.concatenate([np.ldexp(np.float32(1.5), np.arange(-126, 127)), np.ldexp(np.float32(1.0), np.arange(-149, 128))]).astype(np.float32)
    tops = np.concatenate([tops, np.nextafter(tops, np.float32(0)), np.nextafter(tops, np.float32(np.inf))]).astype(np.float32)
    tops = tops[np.isfinite(tops)]
    rng = np.random.default_rng(3)
    X = (tops[:, None] * rng.uniform(-1, 1, (tops.size, 32))).astype(np.float32)
    X[np.arange(tops.size), rng.integers(0, 32, tops.size)] = tops
    for rounding in (0, 1):
        q, t = quantize(G, bnn, X, rounding, 5, True, False)
        got, want = q.get(), mx.quantized(X, rounding, 5)
        n = tops.size * 64
        assert np.array_equal(got[(n + 255) // 256 * 256:], want[(n + 255) // 256 * 256:])
        assert np.array_equal(got[:n], want[:n])
        _, t = quantize(G, bnn, np.ascontiguousarray(X.T), 0, 5, False, True)
        want = mx.quantized(X)
        assert np.array_equal(t.get()[:n], want[:n])


@pytest.mark.parametrize("R,K", SIZES)
def test_dequantize(G, bnn, R, K):
    rng = np.random.default_rng(R + K)
    C = (K + 127) // 128
    codes = rng.integers(0, 16, (R, C * 128))
    e = rng.integers(1, 252, (R, C * 4))
    e[rng.random(e.shape) < 0.05] = 255
    codes[:, K:] = 0
    buf = mx.pack(codes, e)
    for offset in (0, 4):
        q, x = Buffer(buf.size).put(buf), Buffer(R * K * 4, offset)
        bnn.bnn_dequantize_mx4(q.ptr, R, K, x.ptr, G.stream())
        assert np.array_equal(x.get(np.float32).reshape(R, K), mx.unpack(buf, R, K).astype(np.float32), equal_nan=True)


def test_dequantize_scales_from_the_smallest_to_the_largest(G, bnn):
    """Every scale byte with every code: exact, and infinite beyond fp32's range."""
    R, K = 255, 32
    codes = np.zeros((R, 128), np.int64)
    codes[:, :32] = np.arange(32) % 16
    e = np.zeros((R, 4), np.int64)
    e[:, 0] = np.arange(R)
    buf = mx.pack(codes, e)
    q, x = Buffer(buf.size).put(buf), Buffer(R * K * 4)
    bnn.bnn_dequantize_mx4(q.ptr, R, K, x.ptr, G.stream())
    want = mx.unpack(buf, R, K)
    with np.errstate(over="ignore"):
        assert np.array_equal(x.get(np.float32).reshape(R, K), want.astype(np.float32))
    assert np.isfinite(want.astype(np.float32)[:253]).all()


def random_packed(rng, R, K, e_lo=120, e_hi=130, whole=False):
    """A packed matrix with random codes; whole: values that are multiples of 1/4 up to 12."""
    C = (K + 127) // 128
    codes = rng.integers(0, 16, (R, C * 128))
    codes[:, K:] = 0
    e = rng.integers(126, 129, (R, C * 4)) if whole else rng.integers(e_lo, e_hi, (R, C * 4))
    e[:, (K + 31) // 32:] = 0
    return mx.pack(codes, e)


def layer(G, bnn, xq, wq, bias, M, K, N, act, wb=32, offset=0):
    x, w = Buffer(xq.size).put(xq), Buffer(wq.size).put(wq)
    b = Buffer(N * 4, 4).put(bias) if bias is not None else None
    yw = bnn.bnn_packed_words(N, wb)
    y = Buffer(M * yw * wb // 8 if act == bnn.BNN_ACT_SIGN else M * N * 4, offset)
    bnn.bnn_layer_mx4(x.ptr, w.ptr, b.ptr if b else 0, M, K, N, act, wb, y.ptr, G.stream())
    if act == bnn.BNN_ACT_SIGN:
        return y.get(np.uint32 if wb == 32 else np.uint64).reshape(M, yw)
    return y.get(np.float32).reshape(M, N)


LAYERS = [(1, 1, 1), (1, 32, 1), (2, 33, 5), (3, 440, 70), (5, 129, 33), (15, 512, 64), (16, 2048, 100), (17, 130, 257), (31, 96, 31), (33, 1000, 65), (64, 128, 128),
          (65, 256, 129), (100, 3000, 40), (127, 384, 255), (129, 127, 300), (200, 640, 513), (257, 2048, 130), (300, 200, 1003), (520, 1100, 260), (1100, 160, 1100), (3000, 130, 1500), (9000, 128, 1700), (20000, 129, 9), (40, 300, 17000),
          (20000, 64, 1000), (70000, 40, 7), (20, 1100, 130), (50, 2100, 300), (64, 1500, 77),
          (1100, 1500, 3300), (4000, 2050, 1100), (4000, 4000, 1100), (3900, 1025, 3363), (8300, 2500, 4000), (6100, 2000, 8190)]


@pytest.mark.parametrize("M,K,N", LAYERS)
def test_layer_exact_sums(G, bnn, M, K, N):
    """Products that are multiples of 1/16 up to 144: with K up to 4000 every partial sum has at most 24 bits."""
    rng = np.random.default_rng(M * 31 + K * 7 + N)
    xq, wq = random_packed(rng, M, K, whole=True), random_packed(rng, N, K, whole=True)
    bias = (rng.integers(-64, 65, N) / 4).astype(np.float32)
    want = mx.unpack(xq, M, K) @ mx.unpack(wq, N, K).T
    assert np.array_equal(layer(G, bnn, xq, wq, None, M, K, N, bnn.BNN_ACT_LINEAR), want.astype(np.float32))
    h = want + bias
    assert np.array_equal(layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_LINEAR, offset=4), h.astype(np.float32))
    assert np.array_equal(layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_HARDTANH), np.clip(h, -1, 1).astype(np.float32))
    from oracle import oracle as orc
    for wb in (32, 64):
        got = layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_SIGN, wb, offset=wb // 8)
        assert np.array_equal(got, orc.pack_sign(h.astype(np.float32), wb))


@pytest.mark.parametrize("M,K,N", LAYERS)
def test_layer_real_sums(G, bnn, M, K, N):
    rng = np.random.default_rng(M + K + N)
    X = (rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1)))).astype(np.float32)
    W = (rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32)
    xq, wq = mx.quantized(X), mx.quantized(W)
    bias = rng.standard_normal(N).astype(np.float32)
    x, w = mx.unpack(xq, M, K), mx.unpack(wq, N, K)
    h = x @ w.T + bias
    off = K * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + 2.0 ** -23 * (np.abs(h) + np.abs(bias))
    assert (np.abs(layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_LINEAR) - h) <= off).all()
    # (the slope of the sigmoid is at most 1/4; the value's own rounding is half a step)
    got = layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_SIGMOID)
    assert (np.abs(got - 1 / (1 + np.exp(-h))) <= off / 4 + 2.0 ** -24).all()
    # (log sum exp moves by no more than the largest of its arguments does; the rest is fp32 arithmetic on values of this
    # size: exp, a sum of N terms in a few lanes, log and two subtractions, 2^-20 of the largest)
    got = layer(G, bnn, xq, wq, bias, M, K, N, bnn.BNN_ACT_LOGSOFTMAX)
    top = h.max(1, keepdims=True)
    want = h - top - np.log(np.exp(h - top).sum(1, keepdims=True))
    assert (np.abs(got - want) <= off + off.max(1, keepdims=True) + 2.0 ** -20 * (1 + np.abs(h).max(1, keepdims=True) + np.abs(want))).all()


def test_layer_scales_far_apart(G, bnn):
    """Scale bytes over their whole range, the products within fp32's."""
    M, K, N = 40, 256, 70
    rng = np.random.default_rng(0)
    for shift in (0, 60, -60, 100):
        C = 2
        e_x, e_w = rng.integers(110, 140, (M, 4 * C)) + shift, rng.integers(115, 135, (N, 4 * C)) - shift
        xq, wq = mx.pack(rng.integers(0, 16, (M, 128 * C)), e_x), mx.pack(rng.integers(0, 16, (N, 128 * C)), e_w)
        x, w = mx.unpack(xq, M, K), mx.unpack(wq, N, K)
        off = K * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T)
        assert (np.abs(layer(G, bnn, xq, wq, None, M, K, N, bnn.BNN_ACT_LINEAR) - x @ w.T) <= off).all()


@pytest.mark.parametrize("M", [1, 20, 300])
def test_layer_nan_blocks_stay_in_their_rows(G, bnn, M):
    K, N = 300, 150
    rng = np.random.default_rng(M)
    X, W = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    X[M // 2, 170], W[33, 5], W[149, 299] = np.nan, np.inf, np.nan
    xq, _ = quantize(G, bnn, X)
    wq, _ = quantize(G, bnn, W)
    got = layer(G, bnn, xq.get(), wq.get(), None, M, K, N, bnn.BNN_ACT_LINEAR)
    bad = np.zeros((M, N), bool)
    bad[M // 2], bad[:, 33], bad[:, 149] = True, True, True
    assert np.array_equal(np.isnan(got), bad)
    want = mx.unpack(mx.quantized(X), M, K) @ mx.unpack(mx.quantized(W), N, K).T
    assert np.allclose(got[~bad], want[~bad], rtol=1e-4, atol=1e-4)
    bits = layer(G, bnn, xq.get(), wq.get(), None, M, K, N, bnn.BNN_ACT_SIGN)
    assert (bits[M // 2] == 0).all() and not (bits[:, 1] & 2).any()   # Sign of a NaN is -1


@pytest.mark.parametrize("M,K,N", LAYERS + [(1, 2048, 2048), (2, 2048, 2048), (4, 440, 1024), (8, 2049, 333), (48, 1024, 600)])
def test_layer_from_fp32_frames(G, bnn, M, K, N):
    """The same bits as rounding the frames first, wherever the sums are exact; frames whose rows are not 16-byte aligned too."""
    rng = np.random.default_rng(M + 3 * K + 5 * N)
    X = (rng.integers(-6, 7, (M, K)) / 2).astype(np.float32)   # multiples of 1/2 up to 3: the rounded ones are multiples of 1/4
    wq = random_packed(rng, N, K, whole=True)
    bias = (rng.integers(-64, 65, N) / 4).astype(np.float32)
    want = mx.unpack(mx.quantized(X), M, K) @ mx.unpack(wq, N, K).T + bias
    w, b = Buffer(wq.size).put(wq), Buffer(N * 4).put(bias)
    nbytes = bnn.bnn_layer_mx4_realx_workspace_bytes(M, K, N)
    for offset in (0, 4):
        x, ws = Buffer(X.nbytes, offset).put(X), Buffer(nbytes)
        y = Buffer(M * N * 4)
        bnn.bnn_layer_mx4_realx(x.ptr, w.ptr, b.ptr, M, K, N, bnn.BNN_ACT_LINEAR, 32, y.ptr, ws.ptr, nbytes, G.stream())
        assert np.array_equal(y.get(np.float32).reshape(M, N), want.astype(np.float32))
        ws.get()
    yw = bnn.bnn_packed_words(N, 64)
    y = Buffer(M * yw * 8)
    bnn.bnn_layer_mx4_realx(x.ptr, w.ptr, b.ptr, M, K, N, bnn.BNN_ACT_SIGN, 64, y.ptr, ws.ptr, nbytes, G.stream())
    from oracle import oracle as orc
    assert np.array_equal(y.get(np.uint64).reshape(M, yw), orc.pack_sign(want.astype(np.float32), 64))


@pytest.mark.parametrize("M,act", [(1, "linear"), (3, "sigmoid"), (16, "hardtanh"), (40, "logsoftmax"), (200, "linear"), (2, "logsoftmax"), (11, "linear")])
def test_layer_from_fp32_frames_with_real_sums(G, bnn, M, act):
    K, N = 700, 333
    rng = np.random.default_rng(M)
    X = (rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, K)))).astype(np.float32)
    X[M // 2, 64:96] = 0.0
    W = (rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32)
    wq = mx.quantized(W)
    x, w = mx.unpack(mx.quantized(X), M, K), mx.unpack(wq, N, K)
    h = x @ w.T
    off = K * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + 2.0 ** -23 * np.abs(h)
    dx, dw, ws, y = Buffer(X.nbytes).put(X), Buffer(wq.size).put(wq), Buffer(bnn.bnn_layer_mx4_realx_workspace_bytes(M, K, N)), Buffer(M * N * 4)
    bnn.bnn_layer_mx4_realx(dx.ptr, dw.ptr, 0, M, K, N, bnn.ACT_BY_NAME[act], 32, y.ptr, ws.ptr, ws.n, G.stream())
    got = y.get(np.float32).reshape(M, N)
    if act == "sigmoid":
        assert (np.abs(got - 1 / (1 + np.exp(-h))) <= off / 4 + 2.0 ** -24).all()
    elif act == "hardtanh":
        assert (np.abs(got - np.clip(h, -1, 1)) <= off).all()
    elif act == "logsoftmax":
        top = h.max(1, keepdims=True)
        want = h - top - np.log(np.exp(h - top).sum(1, keepdims=True))
        assert (np.abs(got - want) <= off + off.max(1, keepdims=True) + 2.0 ** -20 * (1 + np.abs(h).max(1, keepdims=True) + np.abs(want))).all()
    else:
        assert (np.abs(got - h) <= off).all()


def test_frames_of_inf_and_nan(G, bnn):
    for M in (1, 5, 16, 70):
        K, N = 200, 90
        rng = np.random.default_rng(M)
        X = rng.standard_normal((M, K)).astype(np.float32)
        X[M - 1, 199], X[0, 0] = np.inf, np.nan
        wq = mx.quantized(rng.standard_normal((N, K)).astype(np.float32))
        dx, dw, ws, y = Buffer(X.nbytes).put(X), Buffer(wq.size).put(wq), Buffer(bnn.bnn_layer_mx4_realx_workspace_bytes(M, K, N)), Buffer(M * N * 4)
        bnn.bnn_layer_mx4_realx(dx.ptr, dw.ptr, 0, M, K, N, bnn.BNN_ACT_LINEAR, 32, y.ptr, ws.ptr, ws.n, G.stream())
        nan = np.isnan(y.get(np.float32).reshape(M, N)).all(1)
        assert nan[0] and nan[M - 1] and nan.sum() == len({0, M - 1})


def test_in_graphs_and_on_other_streams(G, bnn):
    """Quantise, layer and the layer from fp32 frames, captured once and replayed on new inputs; and on two streams at once."""
    M, K, N = 70, 500, 300
    rng = np.random.default_rng(9)
    wq = mx.quantized(rng.standard_normal((N, K)).astype(np.float32))
    w = torch.from_numpy(wq).to("cuda:0")
    X = torch.randn((M, K), device="cuda:0")
    q = torch.empty(bnn.bnn_mx4_bytes(M, K), dtype=torch.uint8, device="cuda:0")
    ws = torch.empty(bnn.bnn_layer_mx4_realx_workspace_bytes(M, K, N), dtype=torch.uint8, device="cuda:0")

    def step(X, q, ws, y, z, st):
        bnn.bnn_quantize_mx4(G.ptr(X), M, K, 0, 0, G.ptr(q), 0, st)
        bnn.bnn_layer_mx4(G.ptr(q), G.ptr(w), 0, M, K, N, bnn.BNN_ACT_LOGSOFTMAX, 32, G.ptr(y), st)
        bnn.bnn_layer_mx4_realx(G.ptr(X), G.ptr(w), 0, M, K, N, bnn.BNN_ACT_SIGMOID, 32, G.ptr(z), G.ptr(ws), ws.numel(), st)

    y, z = (torch.empty((M, N), device="cuda:0") for _ in range(2))
    ye, ze = torch.empty_like(y), torch.empty_like(z)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(X, q, ws, y, z, torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        X.copy_(torch.randn((M, K), device="cuda:0"))
        y.zero_(); z.zero_()
        graph.replay()
        step(X, torch.empty_like(q), torch.empty_like(ws), ye, ze, G.stream())
        torch.cuda.synchronize()
        assert torch.equal(y, ye) and torch.equal(z, ze) and torch.isfinite(y).all()
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = [(torch.randn((M, K), device="cuda:0"), torch.empty_like(q), torch.empty_like(ws), torch.empty_like(y), torch.empty_like(z)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, t in zip(streams, sets):
            with torch.cuda.stream(s):
                step(*t, s.cuda_stream)
    torch.cuda.synchronize()
    for t in sets:
        step(t[0], q, ws, ye, ze, G.stream())
        torch.cuda.synchronize()
        assert torch.equal(t[3], ye) and torch.equal(t[4], ze)


def test_matrices_beyond_4_gib(G, bnn):
    """Codes past 2^32 bytes and fp32 past 2^35: the first and the last rows of a matrix of 2^33 + elements, their quantised form and
    their products."""
    R, K, N = (1 << 22) + 37, 2100, 5
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough free memory")
    X = torch.empty((R, K), device="cuda:0")
    X.normal_()
    q = torch.empty(bnn.bnn_mx4_bytes(R, K), dtype=torch.uint8, device="cuda:0")
    assert R * ((K + 127) // 128) * 64 > 1 << 32
    bnn.bnn_quantize_mx4(G.ptr(X), R, K, 1, 77, G.ptr(q), 0, G.stream())
    wq = mx.quantized(np.random.default_rng(0).standard_normal((N, K)).astype(np.float32))
    w = torch.from_numpy(wq).to("cuda:0")
    y = torch.full((R, N), float("nan"), device="cuda:0")
    bnn.bnn_layer_mx4(G.ptr(q), G.ptr(w), 0, R, K, N, bnn.BNN_ACT_LINEAR, 32, G.ptr(y), G.stream())
    some = np.r_[0:40, R // 2:R // 2 + 3, R - 40:R]
    rows = X[torch.from_numpy(some).to("cuda:0")].cpu().numpy()
    key, h = mx.seed_key(77), np.zeros((some.size, K), np.uint32)
    for i, r in enumerate(some):
        h[i] = mx.mix(mx._add(mx.mix(mx._add(key, r)), np.arange(K)))
    x = mx.unpack(mx.pack(*mx.quantize(rows, 1, (h & 0xFFFF) / 65536.0)), some.size, K)
    v = mx.unpack(wq, N, K)
    got = y.cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got[some] - x @ v.T) <= K * 2.0 ** -24 * (np.abs(x) @ np.abs(v).T)).all()
    back = torch.empty((R, K), device="cuda:0") if torch.cuda.mem_get_info()[0] > 40 << 30 else X
    bnn.bnn_dequantize_mx4(G.ptr(q), R, K, G.ptr(back), G.stream())
    assert np.array_equal(back[torch.from_numpy(some).to("cuda:0")].cpu().numpy(), x.astype(np.float32))


def test_layer_of_the_most_outputs(G, bnn):
    """As many outputs as a layer takes (2^22): exact sums at the first, the last and some columns between."""
    M, K, N = 20, 128, 1 << 22
    xq = random_packed(np.random.default_rng(3), M, K, whole=True)
    wq = torch.randint(0, 256, (bnn.bnn_mx4_bytes(N, K),), dtype=torch.uint8, device="cuda:0")
    wq[N * 64:] = 127
    x, y = torch.from_numpy(xq).to("cuda:0"), torch.full((M, N), float("nan"), device="cuda:0")
    bnn.bnn_layer_mx4(G.ptr(x), G.ptr(wq), 0, M, K, N, bnn.BNN_ACT_LINEAR, 32, G.ptr(y), G.stream())
    assert bool(torch.isfinite(y).all())
    at = torch.from_numpy(np.r_[0:70, N // 2 - 40:N // 2 + 40, 64 * 65535 - 40:N]).to("cuda:0")
    n = at.numel()
    some = np.concatenate([wq[:N * 64].view(N, 64)[at].cpu().numpy().reshape(-1), np.zeros(-n * 64 % 256, np.uint8), np.full(4 * n, 127, np.uint8)])
    assert np.array_equal(y[:, at].cpu().numpy(), (mx.unpack(xq, M, K) @ mx.unpack(some, n, K).T).astype(np.float32))
