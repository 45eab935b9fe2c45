"""GPU parity of bnn_update_adamw and bnn_unpack_adamw_states with oracle/mx_oracle.py: fp32 with every operation rounded and
codes that hang on those roundings, so everything is compared bit for bit."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu


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


class Arrays:
    """numpy arrays on the device, each at `shift` bytes past 64-byte alignment, with guards that have to keep their pattern."""

    def __init__(self, arrays, shift=0):
        self.of, self.t = arrays, {}
        for k, a in arrays.items():
            t = torch.full((64 + shift * a.itemsize + a.nbytes + 32,), 0x5A, dtype=torch.uint8, device="cuda:0")
            at = 64 + shift * a.itemsize
            t[at:at + a.nbytes] = torch.from_numpy(a.reshape(-1).view(np.uint8).copy()).to("cuda:0")
            self.t[k] = (t, at)

    def desc(self, clip):
        return {k: t.data_ptr() + at for k, (t, at) in self.t.items()} | {"count": self.of["w"].size, "clip": clip}

    def get(self, k):
        t, at = self.t[k]
        h, a = t.cpu().numpy(), self.of[k]
        assert (h[:at] == 0x5A).all() and (h[at + a.nbytes:] == 0x5A).all(), "written outside " + k
        return h[at:at + a.nbytes].copy().view(a.dtype)


def state(rng, n, bits, fresh):
    f = np.float32
    a = {"w": rng.uniform(-1, 1, n).astype(f), "g": (rng.standard_normal(n) * 1e-3 * np.exp(2 * rng.standard_normal(n))).astype(f)}
    a["g"][rng.random(n) < 0.2] = 0.0
    if bits == 32:
        a["m"] = np.zeros(n, f) if fresh else (rng.standard_normal(n) * 3e-4).astype(f)
        a["v"] = np.zeros(n, f) if fresh else (rng.standard_normal(n) * 1e-3).astype(f) ** 2
    else:
        b = (n + 31) // 32
        a["m"] = np.zeros(n, np.int8) if fresh else rng.integers(-127, 128, n).astype(np.int8)
        a["v"] = np.zeros(n, np.uint8) if fresh else rng.integers(0, 256, n).astype(np.uint8)
        a["m_scale"] = np.zeros(b, np.uint8) if fresh else rng.integers(105, 112, b).astype(np.uint8)
        a["v_scale"] = np.zeros(b, np.uint8) if fresh else rng.integers(105, 112, b).astype(np.uint8)
    return a


def expected(a, bits, step, seed, index, **kw):
    if bits == 32:
        w, m, v, _ = mx.adamw(a["w"], a["g"], a["m"], a["v"], step, **kw)
        return {"w": w, "m": m, "v": v}
    w, m, ms, v, vs = mx.adamw8(a["w"], a["g"], a["m"], a["m_scale"], a["v"], a["v_scale"], step, seed, index, **kw)
    return {"w": w, "m": m, "m_scale": ms, "v": v, "v_scale": vs}


def same(got, want):
    return got.dtype == want.dtype and np.array_equal(got, want, equal_nan=got.dtype.kind == "f")


def params(bnn, bits, step, seed=0, **kw):
    p = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01) | kw
    return bnn.bnn_adamw_params(step=step, state_bits=bits, seed=seed, **p)


COUNTS = [1, 2, 3, 31, 32, 33, 100, 127, 1023, 1024, 1025, 4095, 4096, 4097, 8200, 100003]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 2])
@pytest.mark.parametrize("fresh", [True, False])
def test_update_of_single_tensors(G, bnn, bits, shift, fresh):
    rng = np.random.default_rng(bits + shift)
    for n in COUNTS:
        a = state(rng, n, bits, fresh)
        t = Arrays(a, shift)
        step, seed = (1, 5) if fresh else (77, (n << 40) + 3)
        bnn.bnn_update_adamw(bnn.make_adamw_array([t.desc(n % 2)]), 1, params(bnn, bits, step, seed), G.stream())
        for k, want in expected(a, bits, step, seed, 0, clip=bool(n % 2)).items():
            assert same(t.get(k), want), (n, k)
        assert same(t.get("g"), a["g"])


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_of_every_size_in_one_call(G, bnn, bits):
    """More than one launch takes, empty ones among them; several steps, other hyperparameters."""
    rng = np.random.default_rng(1)
    sizes = [0, 5000, 1, 0, 33] + [int(n) for n in rng.integers(1, 9000, 90)] + [0, 70000, 0]
    arrays = [state(rng, n, bits, True) for n in sizes]
    ts = [Arrays(a, i % 3 if i % 4 == 0 else 0) for i, a in enumerate(arrays)]
    descs = [t.desc(i % 2) if n else {"count": 0} for i, (t, n) in enumerate(zip(ts, sizes))]
    tensors = bnn.make_adamw_array(descs)
    kw = dict(lr=0.02, beta1=0.8, beta2=0.95, eps=1e-6, weight_decay=0.3)
    for step in (1, 2, 3):
        bnn.bnn_update_adamw(tensors, len(sizes), params(bnn, bits, step, step << 33, **kw), G.stream())
        index = 0
        for i, (a, n) in enumerate(zip(arrays, sizes)):
            if n:
                a.update(expected(a, bits, step, step << 33, index, clip=bool(i % 2), **kw))
                index += 1
    for i, (a, t, n) in enumerate(zip(arrays, ts, sizes)):
        for k in a if n else ():
            assert same(t.get(k), a[k]), (i, n, k)


def test_unpack_states(G, bnn):
    rng = np.random.default_rng(4)
    sizes = [int(n) for n in rng.integers(1, 6000, 50)] + [0, 1, 31, 32, 33]
    arrays = [state(rng, n, 8, False) for n in sizes]
    for a in arrays:
        if a["m_scale"].size > 2:
            a["m_scale"][1], a["v_scale"][2] = 255, 0
    for shift in (0, 1):
        ts = [Arrays(a, shift) for a in arrays]
        outs = [Arrays({"w": np.zeros(n, np.float32), "v": np.zeros(n, np.float32)}, shift) for n in sizes]
        tensors = bnn.make_adamw_array([t.desc(0) for t in ts])
        ptrs = [[o.desc(0)[k] for o in outs] for k in ("w", "v")]
        bnn.bnn_unpack_adamw_states(tensors, len(sizes), bnn.make_pointer_array(ptrs[0]), bnn.make_pointer_array(ptrs[1]), G.stream())
        for a, o in zip(arrays, outs):
            r = mx.adamw_decode(a["v"], a["v_scale"])
            assert same(o.get("w"), mx.adamw_decode(a["m"], a["m_scale"])) and same(o.get("v"), r * r)
        # one of the two, and for some tensors neither
        outs = [Arrays({"w": np.zeros(n, np.float32)}, shift) for n in sizes]
        some = [o.desc(0)["w"] if i % 2 else 0 for i, o in enumerate(outs)]
        bnn.bnn_unpack_adamw_states(tensors, len(sizes), None, bnn.make_pointer_array(some), G.stream())
        for i, (a, o) in enumerate(zip(arrays, outs)):
            r = mx.adamw_decode(a["v"], a["v_scale"])
            assert same(o.get("w"), r * r if i % 2 else np.zeros(a["w"].size, np.float32))


@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_out_of_range(G, bnn, bits):
    """Inf, NaN, squares that overflow or vanish: what the formulas give, in 8 bits NaN states for the block, and no other block."""
    rng = np.random.default_rng(6)
    n = 4096 + 50
    a = state(rng, n, bits, False)
    for i, v in enumerate((np.nan, np.inf, -np.inf, 1e25, -1e25, 1e-30, -1e-42, 3e38)):
        a["g"][i * 64 + 7] = v
    a["w"][900:903] = [np.nan, np.inf, -np.inf]
    if bits == 8:
        a["m_scale"][40], a["v_scale"][50] = 255, 255
    t = Arrays(a)
    bnn.bnn_update_adamw(bnn.make_adamw_array([t.desc(1)]), 1, params(bnn, bits, 3, 99), G.stream())
    want = expected(a, bits, 3, 99, 0, clip=True)
    for k in want:
        assert same(t.get(k), want[k]), k


def test_hyperparameters_on_the_device_in_a_graph(G, bnn):
    """A captured update that reads its step and its learning rate from the device, replayed, against eager calls with the same values
    (the step is added to the seed).  A step below 1 counts as 1."""
    for bits in (32, 8):
        rng = np.random.default_rng(bits)
        sizes = [40000, 77]
        arrays = [state(rng, n, bits, True) for n in sizes]
        ts, es = [Arrays(a) for a in arrays], [Arrays(a) for a in arrays]
        graph_list, eager_list = (bnn.make_adamw_array([t.desc(0) for t in s]) for s in (ts, es))
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda:0"), torch.zeros(1, device="cuda:0")
        p = params(bnn, bits, 0, 31, lr_at=lr.data_ptr(), step_at=step.data_ptr())
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            bnn.bnn_update_adamw(graph_list, 2, p, torch.cuda.current_stream().cuda_stream)
        for s in range(1, 6):
            step.fill_(s)
            lr.fill_(np.float32(1e-3) * s)
            graph.replay()
            bnn.bnn_update_adamw(eager_list, 2, params(bnn, bits, s, 31 + s, lr=float(np.float32(1e-3) * np.float32(s))), G.stream())
            torch.cuda.synchronize()
            for t, e, a in zip(ts, es, arrays):
                for k in a:
                    assert same(t.get(k), e.get(k)), (bits, s, k)
        step.fill_(-3)
        graph.replay()
        bnn.bnn_update_adamw(eager_list, 2, params(bnn, bits, 1, 32, lr=float(lr.item())), G.stream())
        torch.cuda.synchronize()
        for t, e, a in zip(ts, es, arrays):
            for k in a:
                assert same(t.get(k), e.get(k)), (bits, k)


@pytest.mark.parametrize("n", [(1 << 32) + 77, (1 << 33) + 3 * 1024 + 77])
def test_more_than_2_to_32_elements(G, bnn, n):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("not enough free memory")
    w, g = (torch.empty(n, device="cuda:0") for _ in range(2))
    w.uniform_(-1, 1)
    g.normal_()
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    ms, vs = (torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    parts = [slice(0, 64), slice((1 << 31) - 32, (1 << 31) + 32), slice((1 << 32) - 64, (1 << 32) + 77), slice(n - 77, n),
             slice((n & ~4095) - 32, (n & ~4095) + 64)]
    parts = [slice(p.start & ~31, p.stop if p.stop == n else p.stop & ~31) for p in parts]
    host = [(w[p].cpu().numpy(), g[p].cpu().numpy()) for p in parts]
    t = bnn.make_adamw_array([dict(w=w.data_ptr(), g=g.data_ptr(), m=m.data_ptr(), v=v.data_ptr(), m_scale=ms.data_ptr(), v_scale=vs.data_ptr(), count=n)])
    bnn.bnn_update_adamw(t, 1, params(bnn, 8, 1, 4), G.stream())
    first = mx.mix(mx._add(mx.mix(mx._add(mx.mix(4), 0)), 0))
    bnn.bnn_unpack_adamw_states(t, 1, bnn.make_pointer_array([g.data_ptr()]), None, G.stream())
    for p, (hw, hg) in zip(parts, host):
        nw, nm, _, r = mx.adamw(hw, hg, np.zeros_like(hw), np.zeros_like(hw), 1)
        b = np.arange(p.start // 32, (p.stop + 31) // 32)
        h = mx.mix(mx._add(mx.mix(mx._add(first, b))[:, None], np.arange(32)[None, :]))
        cm, em = mx.adamw_state(nm, 127.0, (h & 0xFFFF).astype(np.float32))
        cv, ev = mx.adamw_state(r, 255.0, (h >> 16).astype(np.float32))
        bs = slice(b[0], b[-1] + 1)
        assert same(w[p].cpu().numpy(), nw) and same(m[p].cpu().numpy().view(np.int8), cm.astype(np.int8)) and same(v[p].cpu().numpy(), cv.astype(np.uint8))
        assert same(ms[bs].cpu().numpy(), em) and same(vs[bs].cpu().numpy(), ev)
        assert same(g[p].cpu().numpy(), mx.adamw_decode(cm.astype(np.int8), em).astype(np.float32))
