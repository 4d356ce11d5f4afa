"""Host tests of the feed-forward operators: what the entry points refuse (nothing reaches a device: every call here
fails its checks or has no rows), and the pruning of experts."""
import ctypes as C

import numpy as np
import pytest

from paper_2010_16165_amd import binding as B
from paper_2010_16165_amd import experts

ADDR = 1 << 20   # never dereferenced


def mat(rows=4, cols=32, stride=None, dt=B.BF16, ptr=ADDR):
    return B.Matrix(rows, cols, B.min_c_stride(cols, dt) if stride is None else stride, dt, ptr)


def lin(N=16, K=32, dt=B.BF16, act=0, w_stride=None, w=2 * ADDR, w_up=None, bias=None, bias_up=None):
    return B.LinearDesc(N, K, dt, act, B.min_c_stride(K, dt) if w_stride is None else w_stride, w, w_up, bias, bias_up)


def call(op, x, y, res=None):
    return B._lib.fupr_linear_fused(None if op is None else C.byref(op), None if x is None else C.byref(x),
                                    None if res is None else C.byref(res), None if y is None else C.byref(y), None, 0, None)


Y = dict(cols=16, ptr=4 * ADDR)


@pytest.mark.parametrize("status, op, x, y, res", [
    (B.ERR_NULL, None, mat(), mat(**Y), None),
    (B.ERR_NULL, lin(), None, mat(**Y), None),
    (B.ERR_NULL, lin(), mat(), None, None),
    (B.ERR_NULL, lin(w=None), mat(), mat(**Y), None),
    (B.ERR_NULL, lin(), mat(ptr=None), mat(**Y), None),
    (B.ERR_SHAPE, lin(N=0), mat(), mat(**Y), None),
    (B.ERR_SHAPE, lin(K=0), mat(), mat(**Y), None),
    (B.ERR_SHAPE, lin(K=40), mat(), mat(**Y), None),
    (B.ERR_SHAPE, lin(N=24), mat(), mat(**Y), None),
    (B.ERR_SHAPE, lin(), mat(rows=5), mat(**Y), None),
    (B.ERR_SHAPE, lin(), mat(rows=-1), mat(rows=-1, **Y), None),
    (B.ERR_SHAPE, lin(), mat(stride=24), mat(**Y), None),
    (B.ERR_SHAPE, lin(w_stride=24), mat(), mat(**Y), None),
    (B.ERR_SHAPE, lin(), mat(), mat(**Y), mat(rows=3, cols=16, ptr=8 * ADDR)),
    (B.ERR_DTYPE, lin(dt=7), mat(), mat(**Y), None),
    (B.ERR_DTYPE, lin(), mat(dt=B.F16), mat(**Y), None),
    (B.ERR_DTYPE, lin(), mat(), mat(dt=B.F16, **Y), None),
    (B.ERR_DTYPE, lin(), mat(), mat(**Y), mat(cols=16, dt=B.F32, ptr=8 * ADDR)),
    (B.ERR_ALIGN, lin(), mat(stride=36), mat(**Y), None),
    (B.ERR_ALIGN, lin(), mat(ptr=ADDR + 8), mat(**Y), None),
    (B.ERR_ALIGN, lin(w_stride=36), mat(), mat(**Y), None),
    (B.ERR_ALIGN, lin(w=ADDR + 2), mat(), mat(**Y), None),
    (B.ERR_ALIGN, lin(bias=ADDR + 2), mat(), mat(**Y), None),
    (B.ERR_ARG, lin(act=5), mat(), mat(**Y), None),
    (B.ERR_ARG, lin(act=-1), mat(), mat(**Y), None),
    (B.ERR_ARG, lin(bias_up=ADDR), mat(), mat(**Y), None),
    (B.ERR_ARG, lin(), mat(), mat(cols=16, ptr=ADDR + 16), None),              # y over x
    (B.ERR_ARG, lin(), mat(), mat(cols=16, ptr=2 * ADDR + 256), None),         # y over w
    (B.ERR_ARG, lin(), mat(), mat(**Y), mat(cols=16, ptr=4 * ADDR + 32)),      # y over a part of res
    (B.ERR_LIMIT, lin(), mat(stride=1 << 29), mat(**Y), None),
    (B.ERR_LIMIT, lin(), mat(rows=1 << 30, stride=1 << 27), mat(rows=1 << 30, **Y), None),
])
def test_linear_refuses(status, op, x, y, res):
    assert call(op, x, y, res) == status


def test_linear_without_rows_launches_nothing():
    assert call(lin(), mat(rows=0), mat(rows=0, **Y)) == B.FUPR_OK
    assert call(lin(), mat(rows=0, ptr=None), mat(rows=0, cols=16, ptr=None)) == B.FUPR_OK


def test_columns_of_one_buffer_are_apart():
    """x and y side by side in the rows of one buffer share no element; one column over, they do."""
    x, y = mat(rows=0, stride=64), mat(rows=0, cols=16, stride=64, ptr=ADDR + 64)
    assert call(lin(), x, y) == B.FUPR_OK
    for y_ptr, status in ((ADDR + 48, B.ERR_ARG), (ADDR + 112, B.ERR_ARG), (ADDR + 128 * 3 + 48, B.ERR_ARG)):
        assert call(lin(), mat(stride=64), mat(cols=16, stride=64, ptr=y_ptr)) == status, y_ptr


def test_expert_linear_refuses():
    def run(x, y, offsets=ADDR, src=None, E=4, stride=16 * 32, one=None, n_len=None):
        op = B.ExpertLinearDesc(lin() if one is None else one, E, stride, n_len, None)
        return B._lib.fupr_expert_linear_fused(C.byref(op), C.byref(x), offsets, src, C.byref(y), None, 0, None)
    x, y = mat(ptr=16 * ADDR), mat(cols=16, ptr=32 * ADDR)
    assert run(x, y, offsets=None) == B.ERR_NULL
    assert run(x, y, E=0) == B.ERR_SHAPE
    assert run(x, y, stride=-8) == B.ERR_SHAPE
    assert run(x, y, stride=16 * 32 + 4) == B.ERR_ALIGN
    assert run(x, y, offsets=ADDR + 2) == B.ERR_ALIGN
    assert run(x, y, src=ADDR + 1) == B.ERR_ALIGN
    assert run(x, y, n_len=ADDR + 1) == B.ERR_ALIGN
    assert run(mat(rows=3, ptr=16 * ADDR), y) == B.ERR_SHAPE                     # without src the rows match
    assert run(mat(rows=0, ptr=None), y, src=ADDR) == B.ERR_SHAPE
    assert run(x, mat(cols=16, ptr=2 * ADDR + 3 * 1024), src=ADDR) == B.ERR_ARG  # y over the last expert's weights
    assert run(x, y, stride=1 << 45) == B.ERR_LIMIT
    assert run(mat(rows=0), mat(rows=0, cols=16)) == B.FUPR_OK


def test_route_refuses():
    def run(E=8, k=2, score=0, renorm=1, T=4, cols=8, dt=B.F32, ws=None, nws=0, **null):
        r = B.RouterDesc(E, k, score, renorm, 1.0, None, null.pop("bias", None))
        p = {n: ADDR * (i + 2) for i, n in enumerate(("ids", "weights", "offsets", "src", "pos"))}
        p.update(null)
        return B._lib.fupr_moe_route(C.byref(r), C.byref(mat(rows=T, cols=cols, dt=dt)), p["ids"], p["weights"],
                                     p["offsets"], p["src"], p["pos"], ws, nws, None)
    for name in ("ids", "weights", "offsets", "src", "pos"):
        assert run(**{name: None}) == B.ERR_NULL
        assert run(**{name: ADDR + 2}) == B.ERR_ALIGN
    assert run(bias=ADDR + 2) == B.ERR_ALIGN
    assert run(k=0) == run(k=9) == run(E=0) == run(cols=9) == B.ERR_SHAPE
    router = B.RouterDesc(8, 2, 0, 1, 1.0, None, None)

    def logits(dt, stride, ptr):
        return B._lib.fupr_moe_route(C.byref(router), C.byref(mat(rows=0, cols=8, dt=dt, stride=stride, ptr=ptr)), ADDR, ADDR, ADDR,
                                     ADDR, ADDR, None, 0, None)
    assert logits(B.BF16, 9, ADDR + 2) == logits(B.F32, 11, ADDR + 4) == B.FUPR_OK   # rows of any stride
    assert logits(B.BF16, 9, ADDR + 1) == logits(B.F32, 11, ADDR + 2) == B.ERR_ALIGN
    assert logits(B.BF16, 7, ADDR) == B.ERR_SHAPE
    assert run(E=1025, cols=1025) == run(E=64, k=17, cols=64) == B.ERR_LIMIT
    assert run(T=(1 << 31) - 1, k=2) == B.ERR_LIMIT
    assert run(score=2) == run(renorm=2) == B.ERR_ARG
    assert run(dt=9) == B.ERR_DTYPE
    r = B.RouterDesc(8, 2, 0, 1, 1.0, None, None)
    big = int(B._lib.fupr_moe_route_workspace_bytes(C.byref(r), 100000))
    assert big > 0 and B._lib.fupr_moe_route_workspace_bytes(C.byref(r), 4) == 0
    assert run(T=100000) == run(T=100000, ws=ADDR, nws=big - 1) == run(T=100000, ws=ADDR + 16, nws=big) == B.ERR_WORKSPACE


def test_combine_refuses():
    def run(y=None, out=None, res=None, pos=ADDR, weights=ADDR, k=2):
        y = mat(rows=8, ptr=16 * ADDR) if y is None else y
        out = mat(ptr=32 * ADDR) if out is None else out
        return B._lib.fupr_moe_combine(C.byref(y), pos, weights, k, None if res is None else C.byref(res), C.byref(out), None)
    assert run(pos=None) == run(weights=None) == B.ERR_NULL
    assert run(k=0) == run(out=mat(cols=24, ptr=32 * ADDR)) == run(res=mat(rows=5, ptr=64 * ADDR)) == B.ERR_SHAPE
    assert run(out=mat(dt=B.F16, ptr=32 * ADDR)) == run(res=mat(dt=B.F16, ptr=64 * ADDR)) == B.ERR_DTYPE
    assert run(pos=ADDR + 2) == run(out=mat(ptr=32 * ADDR + 8)) == B.ERR_ALIGN
    assert run(out=mat(ptr=16 * ADDR + 64)) == run(res=mat(ptr=32 * ADDR + 64)) == B.ERR_ARG
    assert run(out=mat(rows=0, ptr=None)) == B.FUPR_OK


def test_prune_experts_keeps_the_units_of_largest_norm():
    rng = np.random.default_rng(4)
    E, F, D = 3, 10, 6
    gate, up = (rng.standard_normal((E, F, D)).astype(np.float32) for _ in range(2))
    down = rng.standard_normal((E, D, F)).astype(np.float32)
    rates = [0, 300, 899]
    g, u, d, widths = experts.prune_experts(gate, up, down, rates)
    assert widths.tolist() == [10, 7, 2] and g.shape == (3, 10, 6) and d.shape == (3, 6, 10)
    for e in range(E):
        size = (gate[e].astype(np.float64) ** 2).sum(1) + (up[e].astype(np.float64) ** 2).sum(1)
        keep = np.sort(np.argsort(-size, kind="stable")[:widths[e]])
        assert np.array_equal(g[e, :widths[e]], gate[e][keep])
        assert np.array_equal(u[e, :widths[e]], up[e][keep])
        assert np.array_equal(d[e, :, :widths[e]], down[e][:, keep])
        assert not g[e, widths[e]:].any() and not d[e, :, widths[e]:].any()
    assert experts.prune_experts(gate, up, down, 300)[3].tolist() == [7, 7, 7]
    with pytest.raises(B.FuprError):
        experts.prune_experts(gate, up, down[:, :, :5], 300)
