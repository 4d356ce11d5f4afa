"""GPU tests of the feed-forward operators, each against its definition in 64 bits on the host.

Tolerances are bounds, worked out beforehand.  A sum of K products in fp32 is off by at most 2 K 2^-24 of the sum of
their absolute values (2: the matrix unit need not round each addition to nearest).  An activation multiplies an error
of its argument by at most 1.13 (the steepest slope among them) and adds its own, 2^-18 relative (16-bit results,
hardware 2^v and 1/v; 2^-20 in single precision).  The end is one rounding, half a step of the output's type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f16", "f32"]
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def fx():
    import torch
    from paper_2010_16165_amd import binding as B
    assert torch.cuda.is_available()
    return B, torch


def type_of(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def rows_of(torch, a, dt, pad=0):
    """a on the device, NaN between its rows; rows start at multiples of 16 bytes."""
    unit = 16 // dt.itemsize
    cols = a.shape[-1]
    t = torch.full((*a.shape[:-1], -(-cols // unit) * unit + pad), float("nan"), dtype=dt, device="cuda")
    t[..., :cols] = torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dt)
    return t[..., :cols]


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def act64(name, v):
    from scipy.special import erfc, expit
    if name == "relu":
        return np.maximum(v, 0)
    if name == "silu":
        return v * expit(v)
    if name == "gelu":
        return 0.5 * v * erfc(-v / math.sqrt(2))
    if name == "gelu_tanh":
        return v * expit(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def reference(x, w, b, wu, bu, act, res, out_eps, own):
    """(result, bound on what the kernel's may differ) in 64 bits; own: the activation's own relative error."""
    K = x.shape[1]

    def product(m, bias):
        v, size = x @ m.T, np.abs(x) @ np.abs(m).T
        if bias is not None:
            v, size = v + bias, size + np.abs(bias)
        return v, 2 * (K + 2) * 2.0 ** -24 * size

    h, eh = product(w, b)
    a = act64(act, h)
    ea = eh if act in ("none", "relu") else 1.13 * eh + own * np.abs(a) + 1e-30
    if wu is not None:
        u, eu = product(wu, bu)
        ea = ea * np.abs(u) + np.abs(a) * eu + ea * eu + 2.0 ** -24 * np.abs(a * u)
        a = a * u
    if res is not None:
        a = a + res
        ea = ea + 2.0 ** -24 * np.abs(a)
    tiny = 2.0 ** -25 if out_eps == 2.0 ** -10 else 1e-37   # half the smallest step of fp16
    return a, ea + out_eps / 2 * (np.abs(a) + ea) + tiny


def check(got, want, bound):
    assert got.shape == want.shape
    if not want.size:
        return
    off = np.abs(got - want)
    assert np.isfinite(got).all()
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert (off <= bound).all(), (worst, got[worst], want[worst], bound[worst], float((off > bound).mean()))


SHAPES = [(1, 1, 1), (1, 16, 8), (2, 3, 5), (1, 300, 1000), (5, 64, 64), (7, 33, 200), (16, 130, 257), (17, 48, 72),
          (31, 1000, 96), (33, 65, 64), (64, 128, 128), (65, 257, 129), (100, 20, 520), (128, 64, 2048), (130, 136, 63),
          (255, 256, 192), (257, 300, 136), (300, 40, 1100), (515, 260, 88)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear(fx, shape, dtype):
    """Every size plain, gated, with each activation, with and without bias and residual, outputs of both types."""
    B, torch = fx
    M, N, K = shape
    dt = type_of(torch, dtype)
    rng = np.random.default_rng([M, N, K])
    x = rows_of(torch, rng.standard_normal((M, K)), dt, 16)
    w, wu = (rows_of(torch, rng.standard_normal((N, K)) / math.sqrt(K), dt) for _ in range(2))
    b, bu = (torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda() for _ in range(2))
    for i, act in enumerate(ACTS):
        for gated in (False, True):
            bias, out32, with_res = (i + gated) % 2 == 0, dtype != "f32" and i == 3, i % 3 == 1
            out_t = torch.float32 if out32 else dt
            res = rows_of(torch, rng.standard_normal((M, N)), out_t, 8) if with_res else None
            op = B.Linear(w, b if bias else None, wu if gated else None, bu if gated and bias else None, B.ACTIVATIONS[act])
            y = rows_of(torch, np.full((M, N), 7.0), out_t, 24)
            whole = y.as_strided((M, y.stride(0)), (y.stride(0), 1)) if M > 1 else y
            before = whole[:, N:].clone()
            B.fupr_linear_fused(op, x, y, res, op.workspace(M))
            want, bound = reference(wide(x), wide(w), wide(b) if bias else None, wide(wu) if gated else None,
                                    wide(bu) if gated and bias else None, act, wide(res),
                                    torch.finfo(out_t).eps, 2.0 ** -20 if dtype == "f32" else 2.0 ** -18)
            check(wide(y), want, bound)
            assert torch.equal(whole[:, N:].isnan(), before.isnan())      # between the rows nothing was written


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_in_place_and_in_a_slice(fx, dtype):
    """res is y itself; x, res and y are columns of one buffer."""
    B, torch = fx
    dt = type_of(torch, dtype)
    rng = np.random.default_rng(3)
    M, N, K = 70, 96, 64
    buf = rows_of(torch, rng.standard_normal((M, K + N)), dt)
    w = rows_of(torch, rng.standard_normal((N, K)) / 8, dt)
    x, y = buf[:, :K], buf[:, K:]
    want, bound = reference(wide(x), wide(w), None, None, None, "none", wide(y), torch.finfo(dt).eps, 0)
    op = B.Linear(w)
    B.fupr_linear_fused(op, x, y, y, op.workspace(M))
    check(wide(y), want, bound)


@pytest.mark.parametrize("rows", [1, 9, 40, 200])
def test_what_is_not_finite_stays_where_it_belongs(fx, rows):
    """A NaN in a row of x reaches that row's results only, an infinite weight its own column."""
    B, torch = fx
    N, K = 80, 100
    x = torch.ones((rows, 104), device="cuda", dtype=torch.bfloat16)[:, :K]
    w = torch.ones((N, 104), device="cuda", dtype=torch.bfloat16)[:, :K]
    x[rows // 2, K - 1] = float("nan")
    w[13, 0] = float("-inf")
    for act, at_inf in (("none", -math.inf), ("relu", 0.0), ("silu", math.nan)):
        y = torch.zeros((rows, N), device="cuda", dtype=torch.bfloat16)
        op = B.Linear(w, act=B.ACTIVATIONS[act])
        B.fupr_linear_fused(op, x, y, None, op.workspace(rows))
        v = y.float().cpu().numpy()
        assert np.isnan(v[rows // 2]).all()
        others = np.delete(v, rows // 2, 0)
        assert np.array_equal(others[:, 13], np.full(rows - 1, at_inf, np.float32), equal_nan=True)
        assert np.isfinite(np.delete(others, 13, 1)).all()


def test_linear_far_rows(fx):
    """Rows that lie more than 2^32 bytes apart, in x, in the weights and in y."""
    B, torch = fx
    rng = np.random.default_rng(8)
    for M, N, K, stride in ((70, 20, 40, 1 << 26), (3, 20, 40, 1 << 27)):
        buf = torch.empty(M * stride, dtype=torch.bfloat16, device="cuda")
        x, y = buf.as_strided((M, K), (stride, 1)), buf.as_strided((M, N), (stride, 1), 1 << 20)
        wbuf = torch.empty(N * stride, dtype=torch.bfloat16, device="cuda")
        w = wbuf.as_strided((N, K), (stride, 1))
        x.copy_(torch.from_numpy(rng.standard_normal((M, K))))
        w.copy_(torch.from_numpy(rng.standard_normal((N, K))))
        op = B.Linear(w)
        B.fupr_linear_fused(op, x, y, None, op.workspace(M))
        want, bound = reference(wide(x), wide(w), None, None, None, "none", None, 2.0 ** -7, 0)
        check(wide(y), want, bound)
        # the same rows gathered for one expert, last row first
        src = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda")
        ex = B.ExpertLinear(w[None])
        out = torch.zeros((M, 24), dtype=torch.bfloat16, device="cuda")[:, :N]
        B.fupr_expert_linear_fused(ex, x, torch.tensor([0, M], dtype=torch.int32, device="cuda"), src, out, ex.workspace(M))
        check(wide(out), want[::-1], bound[::-1])
        del buf, wbuf, x, y, w, op, ex


COUNTS = {"even": [16] * 8, "idle": [0, 3, 0, 0, 130, 1, 0, 17], "one": [0, 0, 0, 0, 0, 0, 1, 0], "tall": [700, 0, 5, 300],
          "many": [(7 * e) % 5 for e in range(150)], "first_only": [40, 0, 0]}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("load", COUNTS)
def test_expert_linear(fx, load, dtype):
    """Ragged rows, ragged widths (an expert with none of its filters or inputs among them), with and without src."""
    B, torch = fx
    dt = type_of(torch, dtype)
    counts = COUNTS[load]
    E, total, N, K, T = len(counts), sum(counts), 74, 100, 50
    rng = np.random.default_rng(E)
    spare = 5                                           # rows in front of and behind the experts'
    off = np.concatenate([[0], np.cumsum(counts)]) + spare
    rows = total + 2 * spare
    w, wu = (rows_of(torch, rng.standard_normal((E, N, K)) / 10, dt) for _ in range(2))
    b, bu = (torch.from_numpy(rng.standard_normal((E, N)).astype(np.float32)).cuda() for _ in range(2))
    n_len, k_len = rng.integers(0, N + 1, E), rng.integers(0, K + 1, E)
    n_len[E // 2], k_len[E - 2], n_len[0], k_len[0] = 0, 0, N, K
    offsets = torch.from_numpy(off.astype(np.int32)).cuda()
    for gather in (False, True):
        for act, gated, ragged in (("none", False, False), ("silu", True, True), ("gelu", False, True), ("relu", True, False)):
            x = rows_of(torch, rng.standard_normal((T if gather else rows, K)), dt, 8)
            src = rng.integers(0, T, rows).astype(np.int32)
            src[:spare] = src[total + spare:] = -1      # of rows that belong to nobody
            lens = [torch.from_numpy(v.astype(np.int32)).cuda() if ragged else None for v in (n_len, k_len)]
            op = B.ExpertLinear(w, b if gated else None, wu if gated else None, bu if gated else None, B.ACTIVATIONS[act],
                                *lens)
            y = rows_of(torch, np.full((rows, N), 7.0), dt, 8)
            B.fupr_expert_linear_fused(op, x, offsets, torch.from_numpy(src).cuda() if gather else None, y,
                                       op.workspace(rows))
            got, xs, ws, wus, bs, bus = (wide(t) for t in (y, x, w, wu, b, bu))
            assert (got[:spare] == 7).all() and (got[total + spare:] == 7).all()
            for e, c in enumerate(counts):
                if not c:
                    continue
                n, k = (n_len[e], k_len[e]) if ragged else (N, K)
                at = slice(off[e], off[e + 1])
                xe = (xs[src[at]] if gather else xs[at])[:, :k]
                want, bound = reference(xe, ws[e, :n, :k], bs[e, :n] if gated else None, wus[e, :n, :k] if gated else None,
                                        bus[e, :n] if gated else None, act, None, torch.finfo(dt).eps,
                                        2.0 ** -20 if dtype == "f32" else 2.0 ** -18)
                check(got[at, :n], want, bound)
                assert (got[at, n:] == 0).all()


@pytest.mark.parametrize("rows, n", [(12, 40), (300, 72)])
def test_expert_linear_stays_inside_its_tensors(fx, rows, n):
    """Offsets, src, widths of any content: what they name outside is not touched, and rows that a sane expert has
    and no other claims are right all the same."""
    B, torch = fx
    E, K, T = 4, 64, 20
    rng = np.random.default_rng(1)
    big = torch.full((rows + 64, n + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    y = big[32:32 + rows, :n]
    x = torch.from_numpy(rng.standard_normal((T, K))).to(torch.bfloat16).cuda()
    w = torch.from_numpy(rng.standard_normal((E, n, K))).to(torch.bfloat16).cuda()
    src = torch.full((rows,), 1 << 30, dtype=torch.int32)
    src[:8] = torch.arange(8)
    src[8:] -= torch.arange(rows - 8) * (1 << 22)
    for bad in ([0, 8, -5, 1 << 30, 9], [0, 8, rows + 7, 3, -(1 << 31)], [0, 8, 8, rows * 5, rows * 9]):
        op = B.ExpertLinear(w, n_len=torch.tensor([n, 1 << 30, -1, n + 9], dtype=torch.int32, device="cuda"),
                            k_len=torch.tensor([K, -7, 1 << 30, K + 1], dtype=torch.int32, device="cuda"))
        big.fill_(7.0)
        B.fupr_expert_linear_fused(op, x, torch.tensor(bad, dtype=torch.int32, device="cuda"), src.cuda(), y, op.workspace(rows))
        torch.cuda.synchronize()
        assert (big[:32] == 7).all() and (big[32 + rows:] == 7).all() and (big[:, n:] == 7).all()
        if bad[2] >= 0:
            want, bound = reference(wide(x[:8]), wide(w[0]), None, None, None, "none", None, 2.0 ** -7, 0)
            check(wide(y[:8]), want, bound)


@pytest.fixture(params=range(8), ids=["16x16", "32x32", "32x64", "64x64", "64x128", "128x128", "128x256", "256x256"])
def tile(fx, request):
    """Every call with this tile, whatever the rule would take."""
    B, _ = fx
    B.fupr_tuning_set("linear_tile", str(request.param))
    yield request.param
    B.fupr_tuning_set("linear_tile", None)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_tile(fx, tile, dtype):
    """Reductions that end in the first step, in the second, in the first of a group of waves, and far behind; tiles
    with one row or filter and with all."""
    B, torch = fx
    dt = type_of(torch, dtype)
    eps, own = torch.finfo(dt).eps, 2.0 ** -20 if dtype == "f32" else 2.0 ** -18
    for M, N, K in ((1, 1, 1), (33, 70, 24), (130, 300, 136), (256, 256, 128), (300, 270, 203), (515, 520, 72), (65, 129, 1101),
                    (257, 40, 700)):
        rng = np.random.default_rng([M, N, K])
        x = rows_of(torch, rng.standard_normal((M, K)), dt, 8)
        w, wu = (rows_of(torch, rng.standard_normal((N, K)) / math.sqrt(K), dt) for _ in range(2))
        b, bu = (torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda() for _ in range(2))
        res = rows_of(torch, rng.standard_normal((M, N)), dt)
        for gated in (False, True):
            op = B.Linear(w, b, wu if gated else None, bu if gated else None, B.ACTIVATIONS["silu" if gated else "none"])
            y = rows_of(torch, np.full((M, N), 7.0), dt, 8)
            B.fupr_linear_fused(op, x, y, res, op.workspace(M))
            want, bound = reference(wide(x), wide(w), wide(b), wide(wu) if gated else None, wide(bu) if gated else None,
                                    "silu" if gated else "none", wide(res), eps, own)
            check(wide(y), want, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("load", ["idle", "tall"])
def test_every_tile_of_experts(fx, tile, load, dtype):
    """Ragged rows and widths through src; the lengths of the reduction lie in different steps."""
    B, torch = fx
    dt = type_of(torch, dtype)
    counts = COUNTS[load]
    E, total, N, K, T = len(counts), sum(counts), 270, 210, 60
    rng = np.random.default_rng(E)
    off = np.concatenate([[0], np.cumsum(counts)])
    w, wu = (rows_of(torch, rng.standard_normal((E, N, K)) / 14, dt) for _ in range(2))
    x = rows_of(torch, rng.standard_normal((T, K)), dt)
    n_len, k_len = rng.integers(0, N + 1, E), rng.integers(0, K + 1, E)
    n_len[0], k_len[0] = N, K
    src = rng.integers(0, T, total).astype(np.int32)
    for gated in (False, True):
        op = B.ExpertLinear(w, None, wu if gated else None, None, B.ACTIVATIONS["silu" if gated else "none"],
                            *(torch.from_numpy(v.astype(np.int32)).cuda() for v in (n_len, k_len)))
        y = rows_of(torch, np.full((total, N), 7.0), dt)
        B.fupr_expert_linear_fused(op, x, torch.from_numpy(off.astype(np.int32)).cuda(), torch.from_numpy(src).cuda(), y,
                                   op.workspace(total))
        got, xs, ws, wus = (wide(t) for t in (y, x, w, wu))
        for e in range(E):
            n, k, at = n_len[e], k_len[e], slice(off[e], off[e + 1])
            want, bound = reference(xs[src[at], :k], ws[e, :n, :k], None, wus[e, :n, :k] if gated else None, None,
                                    "silu" if gated else "none", None, torch.finfo(dt).eps,
                                    2.0 ** -20 if dtype == "f32" else 2.0 ** -18)
            check(got[at, :n], want, bound)
            assert (got[at, n:] == 0).all()


def route_reference(logits, k, score, renorm, scale, keep, bias):
    """ids, weights, offsets, src, pos by definition, token by token."""
    T, E = logits.shape
    ids, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        z = logits[t]
        there = np.ones(E, bool) if keep is None else keep != 0
        there = there & ~(z == -np.inf)
        with np.errstate(all="ignore"):
            if score == "softmax":
                most = np.max(z[there]) if there.any() else 0.0
                p = np.where(there, np.exp(z - most), 0.0)
                s = p / p.sum()
            else:
                s = 1 / (1 + np.exp(-z))
        key = z if bias is None else s + bias
        order = sorted((e for e in range(E) if there[e] and not key[e] == -np.inf),
                       key=lambda e: (0 if np.isnan(key[e]) else 1, 0.0 if np.isnan(key[e]) else -key[e], e))[:k]
        ids[t, :len(order)] = order
        v = s[order]
        weights[t, :len(order)] = scale * (v / v.sum() if renorm else v)
    flat = ids.reshape(-1)
    counts = np.bincount(flat[flat >= 0], minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    src, pos = np.full(T * k, -1, np.int32), np.full(T * k, -1, np.int32)
    at = offsets[:-1].copy()
    for s_, e in enumerate(flat):
        if e >= 0:
            src[at[e]], pos[s_] = s_ // k, at[e]
            at[e] += 1
    return ids, weights, offsets, src, pos.reshape(T, k)


def run_route(fx, logits, k, score, renorm, scale=1.0, keep=None, bias=None):
    B, torch = fx
    keep_d = None if keep is None else torch.from_numpy(keep).cuda()
    bias_d = None if bias is None else torch.from_numpy(bias).cuda()
    r = B.Router(logits.shape[1], k, B.SCORES[score], renorm, scale, keep_d, bias_d)
    plan = r.plan(logits.shape[0])
    for t in (plan.ids, plan.src, plan.pos, plan.offsets):
        t.fill_(-77)
    if plan.ws is not None:
        plan.ws.fill_(255)
    B.fupr_moe_route(r, logits, plan)
    return plan


def check_route(plan, want):
    ids, weights, offsets, src, pos = want
    assert np.array_equal(plan.ids.cpu().numpy(), ids)
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    assert np.array_equal(plan.src.cpu().numpy(), src)
    assert np.array_equal(plan.pos.cpu().numpy(), pos)
    got = plan.weights.cpu().numpy().astype(np.float64)
    # exp, the sums of E and of k scores and two divisions in fp32: a few steps each, and E roundings of the sum
    assert np.array_equal(np.isnan(got), np.isnan(weights))
    fine = ~np.isnan(weights)
    assert (np.abs(got - weights)[fine] <= (32 + 2048) * 2.0 ** -24 * np.abs(weights)[fine] + 1e-37).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, E, k", [(1, 1, 1), (1, 8, 2), (5, 64, 8), (3, 60, 6), (33, 128, 8), (64, 96, 3), (65, 7, 7),
                                     (256, 16, 16), (257, 160, 8), (700, 384, 4), (130, 1024, 16), (1500, 65, 1), (20, 513, 9)])
def test_route(fx, T, E, k, dtype):
    B, torch = fx
    rng = np.random.default_rng([T, E, k])
    logits = rows_of(torch, rng.standard_normal((T, E)) * 2, type_of(torch, dtype), 8)
    z = wide(logits)
    bias = (0.2 * rng.standard_normal(E)).astype(np.float32)
    keep = (rng.random(E) < 0.7).astype(np.uint8)
    for score, renorm, b, kp in (("softmax", True, None, None), ("sigmoid", False, None, keep), ("sigmoid", True, bias, None),
                                 ("softmax", False, bias, keep)):
        plan = run_route(fx, logits, k, score, renorm, 1.5, kp, b)
        check_route(plan, route_reference(z, k, score, renorm, 1.5, kp, None if b is None else b.astype(np.float64)))


@pytest.mark.parametrize("T", [9, 300])
@pytest.mark.parametrize("biased", [False, True])
def test_route_ties_masks_and_what_is_not_finite(fx, T, biased):
    B, torch = fx
    E, k = 70, 4
    rng = np.random.default_rng(T)
    z = rng.integers(-2, 3, (T, E)).astype(np.float32)          # full of ties, zeros of both signs
    z[rng.random((T, E)) < 0.1] = -0.0
    z[0] = -np.inf                                              # no expert at all
    z[1] = np.finfo(np.float32).min                             # the type's lowest value is a number
    z[2, 5:] = -np.inf
    z[2, 2:4] = -np.inf                                         # fewer than top_k
    z[3, 11] = np.nan
    z[4] = -np.inf
    z[4, 69] = 0.5
    if not biased:
        z[5, 20] = np.inf
    keep = np.ones(E, np.uint8)
    keep[17] = 0
    z[6, 17] = np.nan                                           # of an expert that is not there
    z[7, 17] = np.inf
    bias = None
    if biased:
        bias = np.zeros(E, np.float32)
        bias[33] = -np.inf
        bias[40] = 0.25
    for score in ("softmax", "sigmoid"):
        plan = run_route(fx, torch.from_numpy(z).cuda()[:, :E].contiguous() if E % 4 == 0 else rows_of(torch, z, torch.float32),
                         k, score, False, 1.0, keep, bias)
        check_route(plan, route_reference(z.astype(np.float64), k, score, False, 1.0, keep,
                                          None if bias is None else bias.astype(np.float64)))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_of_scores_closer_than_32_bits_tell(fx, score):
    """Biases that bring scores of different logits together up to a few times 2^-30: the 64-bit order decides."""
    B, torch = fx
    rng = np.random.default_rng(12)
    T, E, k = 200, 96, 6
    z = np.tile(rng.standard_normal(E), (T, 1)).astype(np.float32)
    s = np.exp(z[0].astype(np.float64))
    s = s / s.sum() if score == "softmax" else s / (1 + s)
    # every biased score lies near 1 / 2, 3 / 4 or 1, as near as a float bias brings it
    bias = (np.array([0.5, 0.75, 1.0])[rng.integers(0, 3, E)] - s).astype(np.float32)
    z[100:, ::7] += (rng.standard_normal((100, len(z[0, ::7]))) * 2.0 ** -20).astype(np.float32)
    plan = run_route(fx, torch.from_numpy(z).cuda(), k, score, True, 1.0, None, bias)
    check_route(plan, route_reference(z.astype(np.float64), k, score, True, 1.0, None, bias.astype(np.float64)))


@pytest.mark.parametrize("dtype", TYPES)
def test_route_of_logits_at_any_stride(fx, dtype):
    """Contiguous rows of 60 or 7 experts, and columns in the middle of wider rows."""
    B, torch = fx
    rng = np.random.default_rng(60)
    for T, E, k in ((1, 60, 8), (6, 60, 4), (333, 60, 8), (70, 7, 3)):
        wide_rows = torch.from_numpy(rng.standard_normal((T, E + 5))).cuda().to(type_of(torch, dtype))
        bias = (0.2 * rng.standard_normal(E)).astype(np.float32)
        for logits in (wide_rows[:, :E].contiguous(), wide_rows[:, 3:E + 3]):
            for b in (None, bias):
                plan = run_route(fx, logits, k, "softmax", True, 1.0, None, b)
                check_route(plan, route_reference(wide(logits), k, "softmax", True, 1.0, None,
                                                  None if b is None else b.astype(np.float64)))


def test_route_without_any_expert(fx):
    B, torch = fx
    for T in (3, 600):
        z = torch.randn((T, 64), device="cuda")
        plan = run_route(fx, z, 2, "softmax", True, 1.0, np.zeros(64, np.uint8), None)
        assert (plan.ids == -1).all() and (plan.weights == 0).all() and (plan.offsets == 0).all()
        assert (plan.src == -1).all() and (plan.pos == -1).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, k, n", [(1, 1, 1), (1, 4, 2048), (3, 8, 100), (50, 5, 77), (33, 16, 264)])
def test_combine(fx, T, k, n, dtype):
    B, torch = fx
    dt = type_of(torch, dtype)
    rng = np.random.default_rng([T, k, n])
    R = T * k + 3
    y = rows_of(torch, rng.standard_normal((R, n)), dt, 8)
    y[0] = float("inf")                                   # of a row that no slot names
    y[1] = float("nan")
    pos = rng.integers(2, R, (T, k)).astype(np.int32)
    pos[rng.random((T, k)) < 0.3] = -1
    pos[rng.random((T, k)) < 0.1] = R                     # outside: adds nothing
    pos[-1] = -1
    w = rng.standard_normal((T, k)).astype(np.float32)
    w[-1] = np.nan                                        # a weight of no row
    pos_d, w_d = torch.from_numpy(pos).cuda(), torch.from_numpy(w).cuda()
    ys, w64 = wide(y), w.astype(np.float64)
    for with_res, in_place in ((False, False), (True, False), (True, True)):
        res = rows_of(torch, rng.standard_normal((T, n)), dt, 16) if with_res else None
        total = wide(res).copy() if with_res else np.zeros((T, n))
        size = np.abs(total)
        for t in range(T):
            for j in range(k):
                if 0 <= pos[t, j] < R:
                    total[t] += w64[t, j] * ys[pos[t, j]]
                    size[t] += np.abs(w64[t, j] * ys[pos[t, j]])
        out = res if in_place else rows_of(torch, np.zeros((T, n)), dt)
        B.fupr_moe_combine(y, pos_d, w_d, res, out)
        bound = 2 * (k + 1) * 2.0 ** -24 * size
        check(wide(out), total, bound + torch.finfo(dt).eps / 2 * (np.abs(total) + bound) + 2.0 ** -25)


def make_layer(torch, dtype, E=12, F=90, D=128, k=3, seed=0, **more):
    from paper_2010_16165_amd import experts
    rng = np.random.default_rng(seed)
    gate, up = (rng.standard_normal((E, F, D)).astype(np.float32) / math.sqrt(D) for _ in range(2))
    down = rng.standard_normal((E, D, F)).astype(np.float32) / math.sqrt(F)
    router = rng.standard_normal((E, D)).astype(np.float32) / math.sqrt(D)
    g, u, d, widths = experts.prune_experts(gate, up, down, [int(p) for p in rng.integers(0, 700, E)])
    return experts.ExpertLayer(router, g, u, d, k, widths, dtype=type_of(torch, dtype), **more), (router, g, u, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 6, 90, 700])
def test_pruned_layer(fx, tokens, dtype):
    """The whole layer of pruned experts against 64 bits, with the experts that the device chose.  Bounds: the hidden
    units and the experts' results are rounded to the type between the operators, half a step each; errors then add as
    sums of absolute values (1.13: the activation's slope, as above)."""
    B, torch = fx
    layer, arrays = make_layer(torch, dtype)
    dt = layer.dtype
    router, g, u, d = (wide(torch.from_numpy(a).to(dt)) for a in arrays)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn((tokens, layer.D), generator=gen, device="cuda").to(dt)
    out = torch.empty_like(x)
    buf = layer.alloc(tokens)
    layer.forward(x, out, buf, x)
    xs, half = wide(x), torch.finfo(dt).eps / 2
    logits = xs @ router.T
    check(wide(buf.logits), logits, 2 * 130 * 2.0 ** -24 * (np.abs(xs) @ np.abs(router).T) + 2.0 ** -24 * np.abs(logits))
    ids, wts = buf.plan.ids.cpu().numpy(), wide(buf.plan.weights)
    want, bound = xs.copy(), np.zeros_like(xs)
    for t in range(tokens):
        for j, e in enumerate(ids[t]):
            h, eh = reference(xs[t:t + 1], g[e], None, u[e], None, "silu", None, 2 * half, 2.0 ** -18)
            y = h @ d[e].T
            ey = eh @ np.abs(d[e]).T + 2 * 92 * 2.0 ** -24 * (np.abs(h) @ np.abs(d[e]).T)
            ey = ey + half * (np.abs(y) + ey)
            want[t] += wts[t, j] * y[0]
            bound[t] += wts[t, j] * (ey[0] + 10 * 2.0 ** -24 * np.abs(y[0]))
    check(wide(out), want, bound + half * (np.abs(want) + bound) + 2.0 ** -24 * np.abs(xs) * 8)


def test_layer_in_a_graph_and_on_another_stream(fx):
    """Captured on a stream of its own and replayed between eager passes: the same bits each time."""
    B, torch = fx
    layer, _ = make_layer(torch, "bf16", seed=5)
    for tokens in (4, 400):
        buf, gbuf = layer.alloc(tokens), layer.alloc(tokens)
        x = torch.zeros((tokens, layer.D), dtype=torch.bfloat16, device="cuda")
        out, gout = torch.empty_like(x), torch.empty_like(x)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.forward(x, gout, gbuf, x)               # (warm)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.forward(x, gout, gbuf, x)
        for i in range(4):
            x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda"))
            layer.forward(x, out, buf, x)
            gout.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, gout)
            assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("rows, n, k", [(1, 4096, 2048), (48, 160, 4096), (512, 1000, 1000)])
def test_linear_gives_the_same_bits_again(fx, rows, n, k):
    B, torch = fx
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, k), generator=gen, device="cuda").to(torch.float16)
    w = torch.randn((n, k), generator=gen, device="cuda").to(torch.float16)
    op = B.Linear(w)
    ws = op.workspace(rows)
    first = torch.empty((rows, n), dtype=torch.float16, device="cuda")
    B.fupr_linear_fused(op, x, first, None, ws)
    for _ in range(5):
        again = torch.full_like(first, float("nan"))
        B.fupr_linear_fused(op, x, again, None, ws)
        assert torch.equal(first, again)
