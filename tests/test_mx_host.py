"""Host-side checks of the 4-bit layers and of the AdamW update that need no GPU: sizes, refusals, and what is launched.
Refused calls are refused before any HIP call (the pointers are made-up addresses that are never dereferenced)."""
import ctypes

import pytest

from test_host_launches import host  # noqa: F401  (the fixture: the library's host side against a stand-in for the HIP runtime)


@pytest.fixture(scope="module")
def bnn():
    import paper_1706_09453_amd as b
    return b


P, Q, R, S, T, U = (0x10000000 * i for i in range(1, 7))


def _status(fn, *a):
    with pytest.raises(Exception) as e:
        fn(*a)
    return e.value.status


def test_sizes(bnn):
    for rows, k in ((1, 1), (1, 128), (3, 129), (64, 440), (4096, 2048), (1 << 22, 2100)):
        chunks = (k + 127) // 128
        assert bnn.bnn_mx4_bytes(rows, k) == (rows * chunks * 64 + 255) // 256 * 256 + rows * chunks * 4
        assert bnn.bnn_layer_mx4_realx_workspace_bytes(rows, k, 7) == bnn.bnn_mx4_bytes(rows, k)
    for rows, k in ((0, 1), (1, 0), (-1, 5), (5, -1), ((1 << 30) + 1, 1), (1, (1 << 30) + 1)):
        assert bnn.bnn_mx4_bytes(rows, k) == 0
    for m, k, n in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (8, (1 << 22) + 1, 8), (8, 8, (1 << 22) + 1), ((1 << 30) + 1, 8, 8)):
        assert bnn.bnn_layer_mx4_realx_workspace_bytes(m, k, n) == 0
    assert ctypes.sizeof(bnn.bnn_adamw_tensor) == 64 and ctypes.sizeof(bnn.bnn_adamw_params) == 80


def test_quantize_refusals(bnn):
    fn = bnn.bnn_quantize_mx4
    assert _status(fn, 0, 4, 64, 0, 0, Q, R) == bnn.BNN_EINVAL
    assert _status(fn, P, 4, 64, 0, 0, 0, 0) == bnn.BNN_EINVAL
    for rounding in (-1, 2):
        assert _status(fn, P, 4, 64, rounding, 0, Q, 0) == bnn.BNN_EINVAL
    for r, c in ((-1, 64), (4, 0), (4, -3), ((1 << 30) + 1, 4), (4, (1 << 30) + 1)):
        assert _status(fn, P, r, c, 0, 0, Q, R) == bnn.BNN_ESHAPE
    assert _status(fn, P + 2, 4, 64, 0, 0, Q, 0) == bnn.BNN_EALIGN
    assert _status(fn, P, 4, 64, 0, 0, Q + 8, 0) == bnn.BNN_EALIGN
    assert _status(fn, P, 4, 64, 0, 0, 0, Q + 8) == bnn.BNN_EALIGN
    assert _status(fn, P, 4, 64, 0, 0, P, 0) == bnn.BNN_EINVAL
    assert _status(fn, P, 4, 64, 0, 0, Q, P + 1008) == bnn.BNN_EINVAL                 # the last 16 bytes of X
    assert _status(fn, P, 4, 64, 0, 0, P - 256 - 16 + 16, 0) == bnn.BNN_EINVAL        # the scale words on X's first bytes
    assert _status(fn, P, 4, 64, 0, 0, Q, Q + 256) == bnn.BNN_EINVAL                  # one form's scales on the other's codes
    assert fn(0, 0, 64, 0, 0, 0, 0) == 0
    fn = bnn.bnn_quantize_mx4_step
    assert _status(fn, P, 4, 64, 0, 0, Q, 0) == bnn.BNN_EINVAL and _status(fn, P, 4, 64, 0, S + 4, Q, 0) == bnn.BNN_EALIGN
    assert _status(fn, P, 4, 64, 0, Q + 8, Q, 0) == bnn.BNN_EINVAL and _status(fn, P, 4, 64, 0, R + 256, 0, R) == bnn.BNN_EINVAL
    assert _status(fn, 0, 4, 64, 0, S, Q, 0) == bnn.BNN_EINVAL and _status(fn, P, 4, 64, 0, S, 0, 0) == bnn.BNN_EINVAL
    assert _status(fn, P, -1, 64, 0, S, Q, 0) == bnn.BNN_ESHAPE and _status(fn, P + 2, 4, 64, 0, S, Q, 0) == bnn.BNN_EALIGN
    assert fn(0, 0, 64, 0, 0, 0, 0) == 0
    fn = bnn.bnn_dequantize_mx4
    assert _status(fn, 0, 4, 64, Q) == bnn.BNN_EINVAL and _status(fn, P, 4, 64, 0) == bnn.BNN_EINVAL
    assert _status(fn, P, -1, 64, Q) == bnn.BNN_ESHAPE and _status(fn, P, 4, 0, Q) == bnn.BNN_ESHAPE
    assert _status(fn, P + 8, 4, 64, Q) == bnn.BNN_EALIGN and _status(fn, P, 4, 64, Q + 2) == bnn.BNN_EALIGN
    assert _status(fn, P, 4, 64, P + 256 + 12) == bnn.BNN_EINVAL                      # on the last scale word
    assert fn(0, 0, 64, 0) == 0


def test_layer_refusals(bnn):
    L, S_ = bnn.BNN_ACT_LINEAR, bnn.BNN_ACT_SIGN
    small, real = bnn.bnn_layer_mx4, bnn.bnn_layer_mx4_realx
    for fn, more in ((small, ()), (real, (T, 1 << 20))):
        def st(x=P, w=Q, b=U, m=4, k=64, n=64, act=L, wb=32, y=R, more=more):
            return _status(fn, x, w, b, m, k, n, act, wb, y, *more)
        assert st(x=0) == st(w=0) == st(y=0) == bnn.BNN_EINVAL
        for act in (-1, bnn.BNN_ACT_RAW_I32, 6):
            assert st(act=act) == bnn.BNN_EINVAL
        assert st(m=-1) == st(k=0) == st(n=0) == st(wb=16) == bnn.BNN_ESHAPE
        assert st(m=(1 << 30) + 1) == st(k=(1 << 22) + 1) == st(n=(1 << 22) + 1) == bnn.BNN_ESHAPE
        assert st(w=Q + 8) == st(b=U + 2) == st(y=R + 2) == st(act=S_, wb=64, y=R + 4) == bnn.BNN_EALIGN
        assert st(y=P) == st(y=Q + 64) == st(y=U) == bnn.BNN_EINVAL
        assert fn(0, 0, 0, 0, 64, 64, L, 32, 0, *((0, 0) if more else ())) == 0
    assert _status(small, P + 8, Q, 0, 4, 64, 64, L, 32, R) == bnn.BNN_EALIGN
    assert _status(real, P + 2, Q, 0, 4, 64, 64, L, 32, R, T, 1 << 20) == bnn.BNN_EALIGN
    need = bnn.bnn_layer_mx4_realx_workspace_bytes(4, 64, 64)
    assert _status(real, P, Q, 0, 4, 64, 64, L, 32, R, T, need - 1) == bnn.BNN_EWORKSPACE
    assert _status(real, P, Q, 0, 4, 64, 64, L, 32, R, 0, need) == bnn.BNN_EWORKSPACE
    assert _status(real, P, Q, 0, 4, 64, 64, L, 32, R, T + 16, need) == bnn.BNN_EALIGN
    for ws in (P, Q, R, U):
        assert _status(real, P, Q, U, 4, 64, 64, L, 32, R, ws, need) == bnn.BNN_EINVAL


def _tensor(bnn, **kw):
    return dict(w=P, g=Q, m=R, v=S, m_scale=T, v_scale=U, count=100, clip=0) | kw


def _params(bnn, **kw):
    return bnn.bnn_adamw_params(**(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, state_bits=32) | kw))


def test_adamw_refusals(bnn):
    def st(p=None, **kw):
        return _status(bnn.bnn_update_adamw, bnn.make_adamw_array([_tensor(bnn, **kw)]), 1, p or _params(bnn))
    nan, inf = float("nan"), float("inf")
    for name in ("w", "g", "m", "v"):
        assert st(**{name: 0}) == bnn.BNN_EINVAL and st(**{name: 0x90000002}) == bnn.BNN_EALIGN
    for name in ("m_scale", "v_scale"):
        assert st(_params(bnn, state_bits=8), **{name: 0}) == bnn.BNN_EINVAL
    assert st(count=-1) == st(count=(1 << 35) + 1) == bnn.BNN_ESHAPE
    assert st(clip=2) == st(clip=-1) == bnn.BNN_EINVAL
    for bad in (dict(lr=-1e-3), dict(lr=nan), dict(lr=inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=0.0),
                dict(eps=1e-50), dict(eps=nan), dict(eps=inf), dict(weight_decay=-1.0), dict(weight_decay=nan), dict(step=0), dict(step=-5), dict(lr=1e30, weight_decay=1e30), dict(lr=1e38, beta1=0.9999), dict(state_bits=16),
                dict(state_bits=0)):
        assert st(_params(bnn, **bad)) == bnn.BNN_EINVAL, bad
    assert st(_params(bnn, lr_at=P + 2)) == st(_params(bnn, step_at=P + 4)) == bnn.BNN_EALIGN
    # what is written on what is read or written
    assert st(g=P) == st(m=P + 396) == st(v=R + 4) == st(g=S) == bnn.BNN_EINVAL
    assert st(_params(bnn, lr_at=P)) == st(_params(bnn, step_at=R + 8)) == bnn.BNN_EINVAL
    eight = _params(bnn, state_bits=8)
    assert st(eight, m_scale=R + 99) == st(eight, v_scale=T + 3) == st(eight, v_scale=Q + 399) == bnn.BNN_EINVAL
    twice = bnn.make_adamw_array([_tensor(bnn), _tensor(bnn, w=0x70000000, m=0x80000000, v=S)])
    assert _status(bnn.bnn_update_adamw, twice, 2, _params(bnn)) == bnn.BNN_EINVAL
    assert _status(bnn.bnn_update_adamw, None, 1, _params(bnn)) == bnn.BNN_EINVAL
    assert _status(bnn.bnn_update_adamw, twice, 2, None) == bnn.BNN_EINVAL
    assert _status(bnn.bnn_update_adamw, twice, -1, _params(bnn)) == bnn.BNN_ESHAPE
    assert bnn.bnn_update_adamw(None, 0, _params(bnn)) == 0
    assert bnn.bnn_update_adamw(bnn.make_adamw_array([{"count": 0}]), 1, _params(bnn)) == 0


def test_unpack_refusals(bnn):
    def st(m_out, v_out, **kw):
        return _status(bnn.bnn_unpack_adamw_states, bnn.make_adamw_array([_tensor(bnn, **kw)]), 1, m_out and bnn.make_pointer_array([m_out]),
                       v_out and bnn.make_pointer_array([v_out]))
    A, B = 0x700000000, 0x800000000
    assert st(None, None) == bnn.BNN_EINVAL
    for name in ("m", "v", "m_scale", "v_scale"):
        assert st(A, B, **{name: 0}) == bnn.BNN_EINVAL
    assert st(A, B, count=-1) == bnn.BNN_ESHAPE
    assert st(A + 2, B) == st(A, B + 1) == bnn.BNN_EALIGN
    assert st(A, A + 396) == st(R, B) == st(A, T - 396) == bnn.BNN_EINVAL
    assert _status(bnn.bnn_unpack_adamw_states, None, -1, None, None) == bnn.BNN_ESHAPE
    assert bnn.bnn_unpack_adamw_states(None, 0, None, None) == 0


def test_launches_of_adamw(host):  # noqa: F811
    """One launch for up to 40 tensors with elements; the largest tensor has a grid that the runtime accepts; a refusal anywhere in the list leaves
    everything undone."""
    got = host("""
def tensors(counts, **kw):
    return bnn.make_adamw_array([dict(w=0x100000000000 * (5 * i + 1), g=0x100000000000 * (5 * i + 2), m=0x100000000000 * (5 * i + 3),
                                      v=0x100000000000 * (5 * i + 4), m_scale=0x100000000000 * (5 * i + 5), v_scale=0x180000000000 + 0x500000000000 * i,
                                      count=c) | kw for i, c in enumerate(counts)])
result = []
for bits in (32, 8):
    p = bnn.bnn_adamw_params(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, state_bits=bits)
    for counts in ([100], [0, 0, 7, 0], [10000] * 40, [10] * 41, [1 << 35], [1 << 35, 5, 1 << 34, 1 << 34, 4096], [0]):
        bnn.bnn_update_adamw(tensors(counts), len(counts), p)
        result.append(launches())
bad = tensors([10] * 100)
bad[99].clip = 3
try:
    bnn.bnn_update_adamw(bad, 100, p)
except bnn.BnnError as e:
    result.append([e.status, len(launches())])
bad = tensors([10] * 100)
bad[99].v = bad[98].w
try:
    bnn.bnn_update_adamw(bad, 100, p)
except bnn.BnnError as e:
    result.append([e.status, len(launches())])
""")
    for half in (got[:7], got[7:14]):
        assert [len(k) for k in half] == [1, 1, 1, 2, 1, 3, 0]
        assert not [l for k in half for l in k if l["wrong"]]
    assert got[14] == [-1, 0] and got[15] == [-1, 0]


def test_launches_of_the_layers(host):  # noqa: F811
    """Every size the layers take has a grid that the runtime accepts; a layer is one launch, log-Softmax a second, rounding the frames one more
    at most."""
    got = host("""
result = []
for act in (bnn.BNN_ACT_LINEAR, bnn.BNN_ACT_SIGN, bnn.BNN_ACT_LOGSOFTMAX):
    for M, K, N in ((1, 1, 1), (1, 2048, 2048), (16, 440, 1024), (17, 440, 1024), (64, 2048, 1 << 22), (65, 1 << 22, 70), (333, 1024, 3307), (4096, 2048, 2048),
                    (16384, 4096, 4096), (1 << 30, 128, 1), (1 << 30, 128, 1000), (5, 128, 1 << 22), (1 << 22, 1 << 22, 1 << 10),
                    (17, 440, 1 << 22), (64, 1024, (1 << 22) - 1), (65, 128, 1 << 22), (300, 128, 1 << 22)):
        bnn.bnn_layer_mx4(A, 1 << 55, 0, M, K, N, act, 32, 1 << 57)
        a = launches()
        need = bnn.bnn_layer_mx4_realx_workspace_bytes(M, K, N)
        bnn.bnn_layer_mx4_realx(A, 1 << 55, 0, M, K, N, act, 32, 1 << 57, 1 << 59, need)
        result.append([act, a, launches()])
for R, C in ((1, 1), (1 << 30, 1), (1, 1 << 30), (1 << 20, 1 << 20), (1 << 30, 1 << 22), (4096, 2048)):
    bnn.bnn_quantize_mx4(A, R, C, 1, 1, 1 << 56, 1 << 58)
    bnn.bnn_dequantize_mx4(1 << 58, R, C, A)
    result.append([-1, launches(), []])
""")
    for act, a, b in got:
        assert not [l for l in a + b if l["wrong"]]
        if act >= 0:
            soft = act == 4
            assert len(a) == 1 + soft and len(b) in (1 + soft, 2 + soft)


def test_sizes_reach_every_tile(host):  # noqa: F811
    """The sizes that the layers are tested at on the device take each of the product's tiles."""
    from test_gpu_mx4 import LAYERS
    got = host("""
result = []
for act in (bnn.BNN_ACT_LINEAR, bnn.BNN_ACT_SIGN):
    for M, K, N in %r:
        bnn.bnn_layer_mx4(A, 1 << 55, 0, M, K, N, act, 32, 1 << 57)
        result.append([act, launches()[0]["kernel"]])
""" % (LAYERS,))
    for act in (1, 3):
        check_tiles([k for a, k in got if a == act])


def check_tiles(got):
    gemm = [k.split("mx4_gemm_kernelI")[1] for k in got if "mx4_gemm_kernel" in k]   # ... activation, a workgroup per CU for all its tiles
    assert {k[20:].split("E")[1] for k in gemm} == {"Lb0", "Lb1"}
    tiles = {k[:20] for k in gemm}
    assert tiles == {"Li1ELi1ELi2ELi2ELi4E", "Li2ELi1ELi2ELi2ELi4E", "Li2ELi2ELi2ELi2ELi3E", "Li2ELi2ELi4ELi2ELi4E", "Li4ELi2ELi2ELi4ELi4E"}
    few = {k.split("mx4_few_kernelI")[1][:4] for k in got if "mx4_few_kernel" in k}
    assert few == {"Li1E", "Li2E", "Li4E"}
