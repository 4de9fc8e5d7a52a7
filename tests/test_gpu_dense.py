"""The workers' dense layer, forward and backward, against float64: ragged groups, shared and own weights, every tile shape, strides, odd sizes,
values that are not finite, and what must be left alone."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2406_05546_b200 import ps
from paper_2406_05546_b200.ps import AdamW, workers_dense_backward, workers_dense_forward, workers_dense_status

gpu = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, 0.0, z)
    if kind == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def matrix(gen, rows, cols, kind, pad=0, scale=1.0, extra=0):
    """[rows + extra, cols] inside a wider buffer whose other values are 77 (extra rows too)."""
    buf = torch.full((rows + extra, cols + pad), 77, dtype=kind, device="cuda")
    buf[:rows, :cols] = (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(kind)
    return buf, buf[:, :cols]


def untouched(buf, rows, cols):
    return bool((buf[rows:] == 77).all() and (buf[:, cols:] == 77).all())


def spans(rows):
    at = 0
    for g, n in enumerate(rows):
        yield g, slice(at, at + n)
        at += n


def sum_error(terms, length, drained):
    """Largest error of a sum of `length` exact products with absolute sum `terms`: an accumulator takes sixteen products at a time and drops less than
    2^-22 of what it holds each time (FP32 results: 32 times at most, then one rounded addition per 512 and per CTA of a cluster)."""
    n = length / 16 + 2
    if drained:
        n = min(n, 34) + length / 512 + 10
    return n * 2.0 ** -22 * terms


def half_step(v, kind):
    """Half the distance of neighbouring values, subnormal ones included."""
    f = torch.finfo(kind)
    return v.abs() * f.eps / 2 + f.smallest_normal * f.eps / 2


# one row each; few rows; ragged with empty groups; one large batch; many single tiles; rows past every tile border
SHAPES = [
    ([1], 1, None, 40, 24),
    ([3, 0, 1, 2], 4, None, 1568, 512),
    ([16, 17, 1, 30], 2, [0, 1, 1, 0], 200, 136),
    ([33, 64, 40], 3, None, 328, 264),
    ([100, 0, 129, 65, 0], 5, None, 136, 200),
    ([128, 129], 1, [0, 0], 520, 128),
    ([300, 257, 511, 90, 700], 2, [0, 0, 1, 1, 0], 96, 1040),
    ([128] * 40, 8, [g % 8 for g in range(40)], 72, 520),
    ([2600], 1, None, 136, 2056),
    ([1000, 0, 1800], 2, [1, 0, 0], 648, 2048),
]


def one_forward(shape, kind, activation, bias, residual, pre, out32, seed=0, pad=(8, 8, 8, 8), extra=0, scale=1.0):
    rows, n_weights, weight_of, K, N = shape
    t, M = TYPES[kind], sum(rows)
    gen = torch.Generator("cuda").manual_seed(seed)
    _, x = matrix(gen, M, K, t, pad[0], scale, extra)
    wbuf = torch.full((n_weights, N, K + pad[1]), 77, dtype=t, device="cuda")
    wbuf[:, :, :K] = (torch.randn(n_weights, N, K, generator=gen, device="cuda") / math.sqrt(K)).to(t)
    w = wbuf[:, :, :K]
    b = torch.randn(n_weights, N, generator=gen, device="cuda").to(t) if bias else None
    _, r = matrix(gen, M, N, t, pad[2]) if residual else (None, None)
    ybuf, y = matrix(gen, M, N, torch.float32 if out32 else t, pad[3], extra=extra)
    pbuf, p = matrix(gen, M, N, t, pad[3], extra=extra) if pre else (None, None)
    assert workers_dense_forward(x, w, rows, weight_of, b, r, activation, y, p) is y
    workers_dense_status()
    assert untouched(ybuf, M, N) and (pbuf is None or untouched(pbuf, M, N))
    for g, s in spans(rows):
        k = weight_of[g] if weight_of else g
        z = x[s].double() @ w[k].double().T
        e = sum_error(x[s].double().abs() @ w[k].double().abs().T, K, out32)
        if bias:
            z = z + b[k].double()
        e = e + z.abs() * 2.0 ** -23
        if pre:
            assert ((p[s].double() - z).abs() <= e + half_step(z.abs() + e, t)).all(), (g, "pre")
        v = act(z, activation)
        e = e * 1.2 + v.abs() * 2.0 ** -20 + 2.0 ** -24 * z.abs()      # |act'| <= 1.13; erf and exp within a few units in the last place
        if residual:
            v = v + r[s].double()
            e = e + v.abs() * 2.0 ** -23
        limit = e + (half_step(v.abs() + e, t) if not out32 else v.abs() * 2.0 ** -23)
        assert ((y[s].double() - v).abs() <= limit).all(), (g, float(((y[s].double() - v).abs() / limit).max()))


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
@pytest.mark.parametrize("kind,activation,bias,residual,pre,out32", [
    ("bf16", "none", False, False, False, False), ("bf16", "relu", True, False, True, False), ("fp16", "gelu", True, True, True, False),
    ("bf16", "silu", False, True, False, True), ("fp16", "none", True, False, False, True)])
def test_forward(shape, kind, activation, bias, residual, pre, out32):
    one_forward(shape, kind, activation, bias, residual, pre, out32)


@gpu
@pytest.mark.parametrize("shape", [([5, 1, 9], 3, None, 37, 51), ([130, 70], 1, [0, 0], 1, 3), ([2600], 1, None, 129, 2051), ([1], 1, None, 7, 1), ([300, 1], 2, None, 65, 9)],
                         ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
@pytest.mark.parametrize("pad", [(0, 0, 0, 0), (1, 2, 3, 5)])
@pytest.mark.parametrize("out32", [False, True])
def test_forward_odd_sizes_and_pitches(shape, pad, out32):
    one_forward(shape, "bf16", "gelu", True, True, True, out32, pad=pad, extra=3)


@gpu
@pytest.mark.parametrize("K", [4096, 16000])
@pytest.mark.parametrize("rows", [[2], [70], [2600]])
def test_forward_long_sums(K, rows):
    one_forward((rows, 1, None, K, 2048), "bf16", "none", True, False, True, True)


def one_backward(shape, kind, activation, add, raw, through, dw32, accumulate=0, pad=(8, 8, 8, 8), extra=0, seed=1, spoil=None):
    rows, n_weights, weight_of, K, N = shape
    t, M, G = TYPES[kind], sum(rows), len(rows)
    d = torch.float32 if dw32 else t
    gen = torch.Generator("cuda").manual_seed(seed)
    _, x = matrix(gen, M, K, t, pad[0], extra=extra)
    _, dy = matrix(gen, M, N, t, pad[1], extra=extra)
    w = (torch.randn(n_weights, N, K + pad[2], generator=gen, device="cuda") / math.sqrt(N)).to(t)[:, :, :K]
    _, da = matrix(gen, M, K, t, pad[3]) if add else (None, None)
    _, xp = matrix(gen, M, K, t, pad[3]) if through else (None, None)
    xbuf, dx = matrix(gen, M, K, t, pad[3], extra=extra) if raw else (None, None)
    pbuf, dp = matrix(gen, M, K, t, pad[0], extra=extra) if through else (None, None)
    wbuf = torch.full((G, N * (K + pad[2]) + 8), 77, dtype=d, device="cuda")
    dw = torch.as_strided(wbuf, (G, N, K), (wbuf.shape[1], K + pad[2], 1))
    bbuf = torch.full((G, N + 8), 77, dtype=d, device="cuda")
    db = bbuf[:, :N]
    if accumulate:
        dw.copy_(torch.randn(G, N, K, generator=gen, device="cuda"))
        db.copy_(torch.randn(G, N, generator=gen, device="cuda"))
    dw0, db0 = dw.double(), db.double()
    if spoil is not None:
        spoil(x, dy, rows)
    workers_dense_backward(dy, x, w, rows, weight_of, xp, activation, da, dx, dp, dw, db, accumulate)
    workers_dense_status()
    for buf in (xbuf, pbuf):
        assert buf is None or untouched(buf, M, K)
    assert (bbuf[:, N:] == 77).all() and (wbuf[:, N * (K + pad[2]):] == 77).all()
    if pad[2]:
        gap = torch.as_strided(wbuf, (G, N, pad[2]), (wbuf.shape[1], K + pad[2], 1), K)
        assert (gap == 77).all()
    for g, s in spans(rows):
        k = weight_of[g] if weight_of else g
        gy, gx = dy[s].double(), x[s].double()
        if spoil is not None and not (torch.isfinite(gy).all() and torch.isfinite(gx).all()):
            continue
        v = gy @ w[k].double()
        e = sum_error(gy.abs() @ w[k].double().abs(), N, False)
        if add:
            v = v + da[s].double()
            e = e + v.abs() * 2.0 ** -23
        if raw:
            assert ((dx[s].double() - v).abs() <= e + half_step(v.abs() + e, t)).all(), (g, "dx")
        if through:
            q = slope(xp[s].double(), activation)
            e2, v2 = e * 1.2 + v.abs() * 2.0 ** -19, v * q      # |act'| <= 1.13, within 2^-20
            assert ((dp[s].double() - v2).abs() <= e2 + half_step(v2.abs() + e2, t)).all(), (g, "dx_pre")
        for got, old, want, terms in ((dw[g], dw0[g], gy.T @ gx, gy.abs().T @ gx.abs()), (db[g], db0[g], gy.sum(0), gy.abs().sum(0))):
            e = sum_error(terms, max(rows[g], 1), dw32)
            if accumulate:
                want = want + old
                e = e + want.abs() * 2.0 ** -23
            limit = e + (half_step(want.abs() + e, t) if not dw32 else want.abs() * 2.0 ** -23)
            assert ((got.double() - want).abs() <= limit).all(), (g, "dw/db", float(((got.double() - want).abs() - limit).max()))


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
@pytest.mark.parametrize("kind,activation,add,raw,through,dw32", [
    ("bf16", "none", False, True, False, False), ("fp16", "relu", True, True, True, True), ("bf16", "gelu", False, False, True, True),
    ("fp16", "silu", True, False, True, False)])
def test_backward(shape, kind, activation, add, raw, through, dw32):
    one_backward(shape, kind, activation, add, raw, through, dw32)


@gpu
@pytest.mark.parametrize("shape", [([5, 1, 9], 3, None, 37, 51), ([130, 70], 1, [0, 0], 1, 3), ([1300], 1, None, 2049, 2051), ([1], 1, None, 7, 1), ([300, 1], 2, None, 65, 9),
                                   ([0, 0], 2, None, 33, 17)], ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
@pytest.mark.parametrize("pad", [(0, 0, 0, 0), (1, 2, 3, 5)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_backward_odd_sizes_and_pitches(shape, pad, accumulate):
    one_backward(shape, "bf16", "gelu", True, True, True, bool(accumulate), accumulate, pad=pad, extra=3)


# rows that start on 16 bytes but not on 32 (pad 0), and on 32 (pad 8), of every persistent tile shape
@gpu
@pytest.mark.parametrize("shape", [([1300, 77, 0, 513, 1, 900], 6, None, 520, 1032), ([2701, 2299], 2, None, 776, 1032), ([1111, 1500], 2, None, 200, 2568)],
                         ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("kind,wide_results", [("bf16", False), ("fp16", True)])
def test_rows_on_sixteen_and_on_thirty_two_bytes(shape, pad, kind, wide_results):
    one_forward(shape, kind, "gelu", True, True, True, wide_results, pad=(pad,) * 4, extra=3)
    one_forward(shape, kind, "relu", False, False, True, wide_results, pad=(pad,) * 4)
    for accumulate in (0, 1):
        one_backward(shape, kind, "silu", True, True, True, wide_results, accumulate, pad=(pad,) * 4, extra=3)


# Every tile shape of every product, with and without its sums handed over on the way (+): the shapes that a device of 148 SMs takes are asked for, so that a
# change of the rules cannot leave one out unseen.  (shape, operands, forward in 16 bits and FP32, input gradient, weight gradient in 16 bits and FP32)
PLANS = [
    (([128, 100, 77, 0, 64] * 12, 60, None, 648, 1032), "bf16", "Single", "Single+", "Single", "Thin", "Thin"),      # many workers on weights of their own
    (([128, 100, 77, 0, 64] * 12, 60, None, 648, 1027), "fp16", "Single", "Single+", "Single", "Thin", "Thin"),
    (([200, 1, 2, 3, 1, 1, 0, 1, 1], 9, None, 520, 264), "bf16", "Few64/4", "Few64+/4", "Few64/2", "Split", "Split"),      # one worker with more rows than a tile has
    (([100, 30, 90, 70, 1, 2, 0, 1], 3, [0, 1, 0, 2, 0, 1, 2, 2], 1096, 328), "fp16", "Few64/8", "Few64+/8", "Few64/2", "Thin", "Thin"),
    (([900, 1000, 530, 1], 4, None, 1288, 1416), "bf16", "Single", "Single+", "Single", "Pair", "Pair+"),
    (([600, 520, 700], 3, None, 1032, 1000), "fp16", "Split", "Split+", "Split", "Single", "Single+"),
    (([2701, 2299], 2, None, 776, 1032), "fp16", "Pair", "Pair+", "Pair", "Split", "Split+"),
    (([1300], 1, None, 8200, 1032), "fp16", "Split+", "Split+", "Pair", "Pair", "Pair+"),      # reductions past 8,192 in FP16
    (([2600], 1, None, 8200, 2056), "fp16", "Pair+", "Pair+", "Pair", "Pair", "Pair+"),
    (([2600], 1, None, 2056, 8200), "fp16", "Pair", "Pair+", "Pair+", "Pair", "Pair+"),
    (([128, 100, 77, 0, 64] * 8, 40, None, 648, 8200), "fp16", "Single", "Single+", "Single+", "Thin", "Thin"),
    (([300], 1, None, 400, 8200), "fp16", "Single", "Single", "Split+/8", "Single", "Single"),
    (([3, 0, 2], 3, None, 8200, 200), "fp16", "Few16+/8", "Few16+/8", "Few16/2", "Thin", "Thin"),
    (([30, 0, 25], 3, None, 8200, 200), "fp16", "Few32+/8", "Few32+/8", "Few32/2", "Thin", "Thin"),
]
plan_id = lambda p: f"{len(p[0][0])}x{sum(p[0][0])}-{p[0][3]}-{p[0][4]}-{p[1]}"


def plan(op, shape, kind, fp32, wide):
    """The tiles that a call takes, and how many CTAs share one."""
    f = ps.load()["_ZN3psk10dense_planEiPKiS1_iiiiiii"]
    f.restype, f.argtypes = C.c_int, [C.c_int, C.c_void_p, C.c_void_p] + [C.c_int] * 7
    rows, _, weight_of, K, N = shape
    r, w = np.array(rows, dtype=np.int32), np.array(weight_of if weight_of else range(len(rows)), dtype=np.int32)
    code = f(op, r.ctypes.data, w.ctypes.data, len(rows), N, K, int(fp32), int(kind == "bf16"), wide, 148)
    return ["Pair", "Single", "Thin", "Split", "Few16", "Few32", "Few64"][code % 16] + ("+" if code & 16 else "") + (f"/{1 << (code >> 5)}" if code >> 5 else "")


@pytest.mark.parametrize("entry", PLANS, ids=plan_id)
@pytest.mark.parametrize("wide", [32, 16, 0])
def test_planned_tiles(entry, wide):
    shape, kind, *want = entry
    got = [plan(0, shape, kind, False, wide), plan(0, shape, kind, True, wide), plan(1, shape, kind, False, wide), plan(2, shape, kind, False, wide), plan(2, shape, kind, True, wide)]
    assert got == want


def test_planned_tiles_leave_no_shape_out():
    seen = {(op, w.split("/")[0]) for _, _, *want in PLANS for op, w in zip("ffxww", want)}
    assert seen >= {(op, name) for op in "fxw" for name in ("Pair", "Pair+", "Single", "Single+", "Split")} | {("w", "Split+"), ("f", "Split+"), ("x", "Split+"), ("w", "Thin")}
    assert seen >= {("f", "Few16+"), ("f", "Few32+"), ("f", "Few64"), ("f", "Few64+"), ("x", "Few16"), ("x", "Few32"), ("x", "Few64")}
    assert plan(0, SHAPES[7], "bf16", False, 32) == plan(0, SHAPES[8], "fp16", True, 0) == "Thin" and plan(0, SHAPES[0], "bf16", False, 32) == "Few16"


@gpu
@pytest.mark.parametrize("entry", PLANS, ids=plan_id)
@pytest.mark.parametrize("pad", [(0, 0, 0, 0), (8, 8, 8, 8), (1, 2, 3, 5)], ids=str)
def test_every_tile_shape(entry, pad):
    shape, kind = entry[:2]
    for wide_results in (False, True):
        one_forward(shape, kind, "gelu", True, True, True, wide_results, pad=pad, extra=3)
        one_backward(shape, kind, "silu", True, True, True, wide_results, accumulate=int(wide_results), pad=pad, extra=3)
    one_forward(shape, kind, "none", False, False, False, False, pad=pad)
    one_backward(shape, kind, "relu", False, True, False, True, pad=pad)


@gpu
@pytest.mark.parametrize("rows", [[70, 5, 0, 33, 200], [1000, 1, 77]])
@pytest.mark.parametrize("N,K", [(136, 200), (2048, 2304)])
@pytest.mark.parametrize("dw32", [False, True])
def test_one_workers_infinities_stay_its_own(rows, N, K, dw32):
    """A worker's NaN and infinities are in none of the other workers' gradients, though their rows share blocks of the reduction."""
    def spoil(x, dy, rows):
        for g, s in spans(rows):
            if g % 2:
                x[s], dy[s] = math.nan, math.inf
    one_backward((rows, len(rows), None, K, N), "bf16", "relu", False, True, True, dw32, spoil=spoil)


@gpu
@pytest.mark.parametrize("shape", [([3, 2], 2, None, 64, 64), ([130, 90], 1, [0, 0], 128, 136)])
def test_values_that_are_not_finite_follow_the_formula(shape):
    rows, n_weights, weight_of, K, N = shape
    x = torch.ones(sum(rows), K, device="cuda").bfloat16()
    w = torch.ones(n_weights, N, K, device="cuda").bfloat16()
    x[0, 0], x[1, 1] = math.nan, math.inf
    for activation in ("none", "relu", "gelu", "silu"):
        y = workers_dense_forward(x, w, rows, weight_of, activation=activation)
        assert torch.isnan(y[0]).all() and (y[1] == math.inf).all() and torch.isfinite(y[2:]).all()
    # a gradient masked by the ReLU is zero, whatever it is
    z = -torch.ones(sum(rows), K, device="cuda").bfloat16()
    dy, dx = torch.full((sum(rows), N), math.inf, device="cuda").bfloat16(), torch.empty_like(z)
    workers_dense_backward(dy, x, w, rows, weight_of, x_pre=z, activation="relu", dx_pre=dx)
    assert not dx.any()


@gpu
def test_empty_call_writes_nothing():
    x, w, y = torch.empty(0, 16, device="cuda").bfloat16(), torch.ones(2, 8, 16, device="cuda").bfloat16(), torch.full((3, 8), 7.0, device="cuda").bfloat16()
    workers_dense_forward(x, w, [0, 0], y=y)
    assert (y == 7).all()
    dw, db = torch.ones(2, 8, 16, device="cuda"), torch.ones(2, 8, device="cuda")
    workers_dense_backward(torch.empty(0, 8, device="cuda").bfloat16(), x, w, [0, 0], dw=dw, db=db, accumulate=True)
    assert (dw == 1).all() and (db == 1).all()
    workers_dense_backward(torch.empty(0, 8, device="cuda").bfloat16(), x, w, [0, 0], dw=dw, db=db)
    assert not dw.any() and not db.any()


@gpu
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[6], SHAPES[8]], ids=lambda s: f"{len(s[0])}x{sum(s[0])}-{s[3]}-{s[4]}")
def test_captured_replayed_and_on_two_streams(shape):
    rows, n_weights, weight_of, K, N = shape
    gen = torch.Generator("cuda").manual_seed(2)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    M = sum(rows)
    x, w, dy = make(M, K), make(n_weights, N, K), make(M, N)

    def both(y, dx, dw, db):
        workers_dense_forward(x, w, rows, weight_of, activation="gelu", y=y)
        workers_dense_backward(dy, x, w, rows, weight_of, dx=dx, dw=dw, db=db)
    outs = [(torch.zeros(M, N, device="cuda").bfloat16(), torch.zeros(M, K, device="cuda").bfloat16(), torch.zeros(len(rows), N, K, device="cuda"),
             torch.zeros(len(rows), N, device="cuda")) for _ in range(4)]
    both(*outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for st, o in zip(streams, outs[1:3]):
            with torch.cuda.stream(st):
                both(*o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(*outs[3])
    for t in outs[3]:
        t.fill_(5)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    workers_dense_status()
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert torch.equal(a, b)
    x.copy_(make(M, K))
    graph.replay()
    both(*outs[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[3]))
    del graph


# The kernels of a backward call run beside one another: what follows the call must find all of them done, and what came before it too.
@gpu
@pytest.mark.parametrize("rows,K,N", [([9, 290, 95, 0, 57, 127], 1568, 512), ([3, 1, 7], 520, 1032), ([4000], 512, 768), ([64] * 12, 264, 520), ([700, 300], 251, 333)],
                         ids=lambda v: str(v) if isinstance(v, int) else f"{len(v)}x{sum(v)}")
@pytest.mark.parametrize("parts", ["db dx dw", "dx dw", "db dw", "db dx"])
def test_nothing_before_or_after_a_backward_call_meets_it(rows, K, N, parts):
    M, G = sum(rows), len(rows)
    gen = torch.Generator("cuda").manual_seed(7)
    x0 = torch.randn(M, K, generator=gen, device="cuda").bfloat16()
    dy0 = torch.randn(M, N, generator=gen, device="cuda").bfloat16()
    w = torch.randn(G, N, K, generator=gen, device="cuda").bfloat16()
    x, dy = torch.empty_like(x0), torch.empty_like(dy0)
    out = {"dx": torch.empty_like(x), "dw": torch.empty(G, N, K, device="cuda"), "db": torch.empty(G, N, device="cuda")}
    out = {k: v for k, v in out.items() if k in parts.split()}
    x.copy_(x0)
    dy.copy_(dy0)
    workers_dense_backward(dy, x, w, rows, **out)
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in out.items()}
    for _ in range(10):
        for v in (x, dy, *out.values()):
            v.fill_(77)
        x.copy_(x0)
        dy.copy_(dy0)
        workers_dense_backward(dy, x, w, rows, **out)
        x.fill_(math.nan)
        dy.fill_(math.nan)
        got = {k: v.clone() for k, v in out.items()}
        workers_dense_status()
        assert all(torch.equal(got[k], want[k]) for k in want)
    # and the next call reads what this one has written
    if "dx" in out:
        x.copy_(x0)
        dy.copy_(dy0)
        y, v = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
        for _ in range(5):
            out["dx"].zero_()
            workers_dense_backward(dy, x, w, rows, **out)
            workers_dense_forward(out["dx"], w, rows, y=y)
        workers_dense_forward(want["dx"], w, rows, y=v)
        workers_dense_status()
        assert torch.equal(y, v)


@gpu
def test_gradients_against_differences():
    """d/dt of sum(c * y(t)) along random directions of x, W and b, y from the forward call in FP32: the differences' error is that of the values
    (2^-22 of the terms' sums, over the step) and the third derivatives' (the layer is linear: none)."""
    rows, K, N = [40, 0, 25], 96, 64
    gen = torch.Generator("cuda").manual_seed(8)
    grid = lambda *s: torch.randint(-8, 9, s, generator=gen, device="cuda").bfloat16() / 8      # sums and differences are exact in bf16
    x, w, b, c = grid(65, K), grid(3, N, K), grid(3, N), grid(65, N)
    dx, dw, db = torch.empty_like(x), torch.empty(3, N, K, device="cuda"), torch.empty(3, N, device="cuda")
    workers_dense_backward(c, x, w, rows, dx=dx, dw=dw, db=db)
    value = lambda x, w, b: float((workers_dense_forward(x, w, rows, bias=b, out_dtype=torch.float32).double() * c.double()).sum())
    ux, uw, ub = grid(65, K), grid(3, N, K), grid(3, N)
    for args, want in (((ux, 0, 0), (dx.double() * ux.double()).sum()), ((0, uw, 0), (dw.double() * uw.double()).sum()), ((0, 0, ub), (db.double() * ub.double()).sum())):
        up, down = (value(x + s * args[0], w + s * args[1], b + s * args[2]) for s in (1, -1))
        size = float((c.double().abs() @ torch.ones(N, 1, device="cuda").double()).sum()) * K * 4
        tol = size * 2.0 ** -22 + (float(dx.double().abs().sum()) * 2.0 ** -9 if args[0] is ux else 0.0)      # dx is rounded to bf16
        assert abs((up - down) / 2 - float(want)) <= tol


@gpu
def test_a_training_step_of_two_layers():
    """Workers with ragged batches and a residual block: forward, backward into one fp32 gradient per worker, their mean, and AdamW with a bf16 copy that the
    next forward reads; against the same in float64 (by autograd), within the roundings of what passes through bf16."""
    rows, D, H = [50, 0, 77, 3], 64, 160
    M, G = sum(rows), 4
    gen = torch.Generator("cuda").manual_seed(9)
    normal = lambda *s, scale=1.0: torch.randn(*s, generator=gen, device="cuda") * scale
    x, target = normal(M, D).bfloat16(), normal(M, D).bfloat16()
    master = [normal(H, D, scale=0.1), normal(H, scale=0.1), normal(D, H, scale=0.1), normal(D, scale=0.1)]
    copies = [p.bfloat16() for p in master]
    per_worker = [torch.empty(G, *p.shape, device="cuda") for p in master]
    mean = [torch.empty_like(p) for p in master]
    opt = AdamW(master, mean, copies=copies, weight_decay=0.0)
    for step in (1, 2):
        w1, b1, w2, b2 = copies
        pre, h, y = torch.empty(M, H, device="cuda").bfloat16(), None, None
        one = [0] * G
        h = workers_dense_forward(x, w1, rows, one, bias=b1, activation="gelu", pre=pre)
        y = workers_dense_forward(h, w2, rows, one, bias=b2, residual=x)
        dy = (y.float() - target.float()).bfloat16()
        dpre, dx = torch.empty_like(pre), torch.empty_like(x)
        workers_dense_backward(dy, h, w2, rows, one, x_pre=pre, activation="gelu", dx_pre=dpre, dw=per_worker[2], db=per_worker[3])
        workers_dense_backward(dpre, x, w1, rows, one, dx_add=dy, dx=dx, dw=per_worker[0], db=per_worker[1])
        ref = [p.double().requires_grad_() for p in copies] + [x.double().requires_grad_()]
        z = ref[4] @ ref[0].T + ref[1]
        out = act(z, "gelu") @ ref[2].T + ref[3] + ref[4]
        (0.5 * (out - target.double()).square()).sum().backward()
        got = [t.sum(0).double() for t in per_worker] + [dx.double()]
        for a, r in zip(got, ref):      # five roundings to bf16 on the way (pre, h, y, dy, dpre), each 2^-9 at most of what it rounds
            assert float((a - r.grad).norm() / r.grad.norm()) < 5 * 2.0 ** -9
        for m, t in zip(mean, per_worker):
            torch.mean(t, 0, out=m)
        opt.ps_adamw_step(lr=1e-2, step=step)
        torch.cuda.synchronize()
        assert all(torch.equal(c, p.bfloat16()) for c, p in zip(copies, master))


@gpu
@pytest.mark.parametrize("N", [256, 250, 251])
@pytest.mark.parametrize("rows", [[5, 2], [140, 60], [2600]])
def test_the_added_gradient_may_lie_where_the_result_goes(rows, N):
    gen = torch.Generator("cuda").manual_seed(4)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    K, M, G = N, sum(rows), len(rows)
    x, w, dy, extra, z = make(M, K), make(G, N, K), make(M, N), make(M, K), make(M, K)
    apart, apart_pre, pre = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    workers_dense_backward(dy, x, w, rows, x_pre=z, activation="silu", dx_add=extra, dx=apart, dx_pre=apart_pre)
    workers_dense_backward(dy, x, w, rows, x_pre=z, activation="silu", dx_add=extra, dx=extra, dx_pre=pre)
    assert torch.equal(apart, extra) and torch.equal(apart_pre, pre)


@gpu
@pytest.mark.parametrize("entry", PLANS + [((rows, len(rows), None, K, N), "bf16") for rows, K, N in (([5, 2], 264, 250), ([140, 60], 264, 251), ([2600], 136, 2056))], ids=plan_id)
def test_the_residual_may_lie_where_the_result_goes(entry):
    (rows, n_weights, weight_of, K, N), t = entry[0], TYPES[entry[1]]
    gen = torch.Generator("cuda").manual_seed(4)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(t)
    M = sum(rows)
    for width in (N, N + 8 if N % 8 == 0 else N):
        x, w, both, pre = make(M, K), make(n_weights, N, K), make(M, width)[:, :N], torch.empty(M, N, device="cuda", dtype=t)
        apart = workers_dense_forward(x, w, rows, weight_of, residual=both.clone(), activation="gelu", pre=pre)
        assert workers_dense_forward(x, w, rows, weight_of, residual=both, activation="gelu", y=both, pre=pre) is both
        assert torch.equal(apart, both)


@gpu
def test_odd_sizes_captured_and_replayed():
    """Operands that are laid out anew: the workspace is the graph's own."""
    gen = torch.Generator("cuda").manual_seed(5)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    rows, K, N = [33, 0, 150], 77, 91
    x, w, dy = make(183, K), make(3, N, K), make(183, N)
    y, dx, dw, db = make(183, N), make(183, K), torch.zeros(3, N, K, device="cuda"), torch.zeros(3, N, device="cuda")

    def call():
        workers_dense_forward(x, w, rows, y=y)
        workers_dense_backward(dy, x, w, rows, dx=dx, dw=dw, db=db)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        x.copy_(make(183, K))
        w.copy_(make(3, N, K))
        graph.replay()
        other = torch.randn(1 << 20, device="cuda")      # other work in memory that the calls outside the graph had
        got = [t.clone() for t in (y, dx, dw, db)]
        call()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw, db)))
        del other
    del graph


@gpu
@pytest.mark.parametrize("K,N", [(16, 32768), (24, 32774)])
def test_offsets_past_32_bits(K, N):
    """Results of more than 2^31 elements: the last rows, and those on either side of the 2^31st element."""
    M = (1 << 31) // N + 300
    gen = torch.Generator("cuda").manual_seed(6)
    x, w = torch.randn(M, K, generator=gen, device="cuda").bfloat16(), torch.randn(1, N, K, generator=gen, device="cuda").bfloat16()
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    workers_dense_forward(x, w, [M], y=y)
    edge = (1 << 31) // N
    for r in (slice(0, 3), slice(edge - 2, edge + 2), slice(M - 3, M)):
        want = x[r].double() @ w[0].double().T
        e = sum_error(x[r].double().abs() @ w[0].double().abs().T, K, False)
        assert ((y[r].double() - want).abs() <= e + half_step(want.abs() + e, torch.bfloat16)).all()
    # and read: a gradient whose rows lie that far out
    dx = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    workers_dense_backward(y, x, w, [M], dx=dx)
    r = slice(M - 3, M)
    want = y[r].double() @ w[0].double()
    e = sum_error(y[r].double().abs() @ w[0].double().abs(), N, False)
    assert ((dx[r].double() - want).abs() <= e + half_step(want.abs() + e, torch.bfloat16)).all()


@gpu
def test_weight_gradients_past_32_bits():
    """A gradient per worker, the last one's beyond the 2^31st element."""
    G, N, K = 9, 16384, 16384
    gen = torch.Generator("cuda").manual_seed(7)
    x, dy = torch.randn(G, K, generator=gen, device="cuda").bfloat16(), torch.randn(G, N, generator=gen, device="cuda").bfloat16()
    w, dw = torch.empty(1, N, K, dtype=torch.bfloat16, device="cuda"), torch.empty(G, N, K, dtype=torch.bfloat16, device="cuda")
    workers_dense_backward(dy, x, w, [1] * G, weight_of=[0] * G, dw=dw)
    for g in (0, G - 1):
        want = dy[g].double()[:, None] * x[g].double()[None, :256]
        assert ((dw[g][:, :256].double() - want).abs() <= half_step(want, torch.bfloat16) * 1.01).all()
        want = dy[g].double()[-64:, None] * x[g].double()[None]
        assert ((dw[g][-64:].double() - want).abs() <= half_step(want, torch.bfloat16) * 1.01).all()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("activation", ["gelu", "silu"])
def test_activations_keep_their_digits(kind, activation):
    """The values of a 16-bit type through an identity matrix: a sum is one product and exact, so that only the activation's own error is left, within what the
    header states (relative, in the tails too)."""
    t = TYPES[kind]
    z = torch.arange(65536, device="cuda").to(torch.int32).to(torch.int16).view(t)
    z = z[torch.isfinite(z) & (z.abs() < 1000)]
    z = torch.cat([z, z.new_zeros(-z.numel() % 64)]).view(-1, 64)
    M = z.shape[0]
    eye, rows = torch.eye(64, device="cuda", dtype=t).view(1, 64, 64), [M]
    y = workers_dense_forward(z, eye, rows, activation=activation, out_dtype=torch.float32)
    zd = z.double()
    want = act(zd, activation)
    grow = zd.square() if activation == "gelu" else zd.abs()
    assert ((y.double() - want).abs() <= want.abs() * (2.0 ** -19 + grow * 2.0 ** -22) + 2.0 ** -110).all()
    # the derivative, through a gradient of one: its 16-bit result is rounded once
    dy, dz = torch.zeros(M, 64, device="cuda", dtype=t), torch.empty_like(z)
    workers_dense_backward(dy, z, eye, rows, x_pre=z, activation=activation, dx_add=torch.ones_like(z), dx_pre=dz)
    workers_dense_status()
    want = slope(zd, activation)
    e = 2.0 ** -20 + 2.0 ** -22 * zd.abs()
    assert ((dz.double() - want).abs() <= e + half_step(want.abs() + e, t)).all()


def backward_within(limit, dy, x, w, rows, dw):
    """dw of a backward call whose waits end after `limit` clocks."""
    counts, G, N, K = np.array(rows, dtype=np.int32), len(rows), dy.shape[1], x.shape[1]
    kind = {torch.bfloat16: ps.TYPE_BF16, torch.float16: ps.TYPE_FP16, torch.float32: ps.TYPE_FP32}
    shared = np.zeros(G, dtype=np.int32)
    l = ps.DenseLayer(G, 1, counts.ctypes.data, shared.ctypes.data, K, N, kind[x.dtype], 0, x.data_ptr(), x.stride(0), w.data_ptr(), K, N * K, None, 0,
                      torch.cuda.current_stream().cuda_stream)
    out = ps.DenseGradients(dy=dy.data_ptr(), dy_pitch=dy.stride(0), dw=dw.data_ptr(), dw_pitch=K, dw_stride=N * K, dw_type=kind[dw.dtype])
    assert ps.load().workers_dense_selftest_backward(C.byref(l), C.byref(out), limit) == 0
    workers_dense_status()


@gpu
@pytest.mark.parametrize("kind,result", [("bf16", torch.float32), ("fp16", torch.float16)])
def test_no_wait_grows_with_the_work(kind, result):
    """A worker of 2^19 rows, some five million clocks of products to a pair of CTAs, ahead of one whose last block is ragged: no single wait takes 600,000."""
    rows, N, K = [1 << 19, 100], 1792, 1792
    gen = torch.Generator("cuda").manual_seed(11)
    x, dy = ((torch.randn(sum(rows), c, generator=gen, device="cuda", dtype=TYPES[kind]) * 0.25) for c in (K, N))
    w = torch.empty(N, K, device="cuda", dtype=TYPES[kind])
    dw = torch.full((2, N, K), 77, device="cuda", dtype=result)
    backward_within(600000, dy, x, w, rows, dw)
    for g, s in spans(rows):
        cols = slice(0, K) if g else slice(K - 32, K)
        gy, gx = dy[s].double(), x[s, cols].double()
        want, e = gy.T @ gx, sum_error(gy.abs().T @ gx.abs(), rows[g], result == torch.float32)
        limit = e + (want.abs() * 2.0 ** -23 if result == torch.float32 else half_step(want.abs() + e, result))
        assert ((dw[g][:, cols].double() - want).abs() <= limit).all(), g


@gpu
def test_a_wait_that_gave_up_is_reported_to_every_thread_once():
    """A thread that asks takes the answer from no other, and failures that come later are reported anew."""
    from concurrent.futures import ThreadPoolExecutor

    def ask():
        try:
            workers_dense_status()
        except ps.PSError as e:
            assert "PS_ERR_DEVICE_STATUS" in str(e)
            return True
        return False
    side = torch.cuda.Stream()
    with ThreadPoolExecutor(1) as one, ThreadPoolExecutor(1) as two:
        for pool in (one, two):
            pool.submit(ask).result()
        ask()
        assert not ask() and not one.submit(ask).result()
        for stream in (torch.cuda.current_stream(), side):
            assert ps.load().workers_dense_selftest_wait_timeout(10000, stream.cuda_stream) == 0
            torch.cuda.synchronize()
            assert one.submit(ask).result() and ask() and two.submit(ask).result()
            assert not ask() and not two.submit(ask).result() and not one.submit(ask).result()
    # and the next call is as good as any
    x, w = torch.ones(3, 16, device="cuda").bfloat16(), torch.ones(1, 8, 16, device="cuda").bfloat16()
    assert (workers_dense_forward(x, w, [3]) == 16).all()
    workers_dense_status()


# Sums of one sign so long that an accumulator's truncation would come near the result's rounding and pass it.  An instruction cuts its sixteen products and the
# accumulator at 2^-25 of a power of two that is not above their sum: half of that each in the mean, 17 / 2 * 2^-25 of the partial sum, and half as much
# of the whole, since partial sums grow evenly: n instructions lose 17 / 4 * 2^-25 n of it.  (Measured, of 1,024: 1.04e-4, where this gives 1.3e-4.)
# It is the same for all results while their roundings average out (rows and columns differ in scale), so the mean of the relative errors shows it.  An accumulator takes 512 (FP16) or
# 4,096 (BF16) at most; the mean of n roundings, each within half a step u and evenly spread, has a deviation of u / sqrt(3 n).
LONG_SUMS = [("dw", "fp16", 1 << 18, 1664, 1664), ("dw", "fp16", 1 << 18, 2304, 2304), ("dw", "fp16", 1 << 21, 64, 72), ("dw", "bf16", 1 << 21, 1664, 1664),
             ("forward", "fp16", 2600, 2048, 1 << 18), ("forward", "fp16", 600, 1040, 1 << 18), ("forward", "fp16", 3, 520, 1 << 20),
             ("dx", "fp16", 2600, 1 << 18, 2048), ("dx", "fp16", 600, 1 << 18, 1040), ("dx", "fp16", 3, 1 << 20, 520), ("dx", "bf16", 2600, 1 << 20, 2048)]


@gpu
@pytest.mark.parametrize("op,kind,M,N,K", LONG_SUMS)
def test_long_sums_keep_their_low_bits(op, kind, M, N, K):
    t = TYPES[kind]
    gen = torch.Generator("cuda").manual_seed(12)
    def positive(*s, scaled):      # along dimension `scaled` the values differ in scale
        shape = [1] * len(s)
        shape[scaled] = s[scaled]
        return (torch.rand(*s, generator=gen, device="cuda", dtype=t) * 0.0625 + 0.03125) * (0.5 + 0.5 * torch.rand(*shape, generator=gen, device="cuda")).to(t)
    length = {"dw": M, "forward": K, "dx": N}[op]
    if op == "dw":
        x, dy, w = positive(M, K, scaled=1), positive(M, N, scaled=1), torch.empty(1, N, K, device="cuda", dtype=t)
        got = torch.empty(1, N, K, device="cuda", dtype=t)
        workers_dense_backward(dy, x, w, [M], dw=got)
        got, left, right = got[0, :, -512:], dy.T, x[:, -512:]
    elif op == "forward":
        x, w = positive(M, K, scaled=0), positive(1, N, K, scaled=1)
        got = workers_dense_forward(x, w, [M])
        got, left, right = got[:, -512:], x, w[0, -512:].T
    else:
        dy, w = positive(M, N, scaled=0), positive(1, N, K, scaled=2)
        got = torch.empty(M, K, device="cuda", dtype=t)
        workers_dense_backward(dy, torch.empty(M, K, device="cuda", dtype=t), w, [M], dx=got)
        got, left, right = got[:, -512:], dy, w[0, :, -512:]
    workers_dense_status()
    want = torch.zeros(got.shape, device="cuda", dtype=torch.float64)
    for a in range(0, length, 1 << 16):
        want += left[:, a:a + (1 << 16)].double() @ right[a:a + (1 << 16)].double()
    assert torch.isfinite(got).all()
    off = (got.double() - want) / want
    u = torch.finfo(t).eps / 2
    lost = 17 / 4 * 2.0 ** -25 * {"fp16": 512, "bf16": 4096}[kind]
    assert (off.abs() <= u + 2 * lost).all()
    assert abs(float(off.mean())) <= lost + 6 * u / math.sqrt(3 * off.numel())


# ---- refusals --------------------------------------------------------------------------------------------------------------
def layer(**more):
    """A layer whose addresses are never read: every refusal comes before any launch."""
    rows = np.array(more.pop("row_list", [4, 0, 3]), dtype=np.int32)
    l = ps.DenseLayer(len(rows), 3, rows.ctypes.data, None, 32, 16, ps.TYPE_BF16, 0, 1 << 20, 32, 1 << 21, 32, 512, None, 0, None)
    l._keep = rows
    for k, v in more.items():
        if k == "weight_list":
            l._w = np.array(v, dtype=np.int32)
            l.weight_of = l._w.ctypes.data
        else:
            setattr(l, k, v)
    return l


BAD_LAYERS = [dict(groups=0), dict(groups=257), dict(rows=None), dict(row_list=[4, -1, 3]), dict(row_list=[2**31 - 1, 2**31 - 1, 1]), dict(n_weights=2), dict(n_weights=0),
              dict(weight_list=[0, 1, 3]), dict(weight_list=[0, -1, 0]), dict(type=ps.TYPE_FP32), dict(type=7), dict(in_features=0), dict(out_features=-1),
              dict(in_features=(1 << 20) + 1), dict(activation=4), dict(activation=-1), dict(x=None), dict(x_pitch=31), dict(weight=None), dict(weight_pitch=31),
              dict(weight_stride=511), dict(x=(1 << 20) + 1)]


@pytest.mark.parametrize("bad", BAD_LAYERS, ids=str)
def test_refused_layers(bad):
    lib, size = ps.load(), C.c_uint64()
    out = ps.DenseOutput(y=1 << 22, y_pitch=16, y_type=ps.TYPE_BF16)
    grads = ps.DenseGradients(dy=1 << 22, dy_pitch=16, dx=1 << 23, dx_pitch=32, dw_type=ps.TYPE_FP32)
    l = layer(**bad)
    assert lib.workers_dense_forward(C.byref(l), C.byref(out)) == -1
    assert lib.workers_dense_backward(C.byref(l), C.byref(grads)) == -1
    assert lib.workers_dense_workspace(C.byref(l), None, 0, C.byref(size)) == -1


@pytest.mark.parametrize("bad", [dict(y=None), dict(y_pitch=15), dict(y_type=ps.TYPE_FP16), dict(y_type=9), dict(y=(1 << 22) + 1), dict(residual=1 << 23, residual_pitch=15),
                                 dict(pre=1 << 23, pre_pitch=1), dict(bias=1 << 23, bias_stride=15), dict(bias=(1 << 23) + 1, bias_stride=16)], ids=str)
def test_refused_outputs(bad):
    out = ps.DenseOutput(y=1 << 22, y_pitch=16, y_type=ps.TYPE_BF16)
    for k, v in bad.items():
        setattr(out, k, v)
    assert ps.load().workers_dense_forward(C.byref(layer()), C.byref(out)) == -1


@pytest.mark.parametrize("bad", [dict(dy=None), dict(dy_pitch=15), dict(dx_pitch=31), dict(dx_pre=1 << 23, dx_pre_pitch=32), dict(dw=1 << 23, dw_pitch=31, dw_stride=512),
                                 dict(dw=1 << 23, dw_pitch=32, dw_stride=511), dict(db=1 << 23, db_stride=15), dict(dw_type=ps.TYPE_FP16), dict(accumulate=2),
                                 dict(dw=(1 << 23) + 2, dw_pitch=32, dw_stride=512), dict(dx_add=1 << 23, dx_add_pitch=3)], ids=str)
def test_refused_gradients(bad):
    grads = ps.DenseGradients(dy=1 << 22, dy_pitch=16, dx=1 << 23, dx_pitch=32, dw_type=ps.TYPE_FP32)
    for k, v in bad.items():
        setattr(grads, k, v)
    assert ps.load().workers_dense_backward(C.byref(layer()), C.byref(grads)) == -1


def test_refused_limits():
    for limit in (0, -1, 2000000001):
        assert ps.load().workers_dense_selftest_backward(C.byref(layer()), C.byref(ps.DenseGradients()), limit) == -1
        assert ps.load().workers_dense_selftest_wait_timeout(limit, None) == -1


def test_workspace_is_asked_for_where_tile_copies_cannot_read():
    lib, size = ps.load(), C.c_uint64()
    ask = lambda l, dy=None, pitch=0: lib.workers_dense_workspace(C.byref(l), dy, pitch, C.byref(size)) == 0 and size.value
    assert ask(layer()) == 0 and ask(layer(), 1 << 22, 16) == 0
    assert ask(layer(x_pitch=33)) >= 7 * 32 * 2 and ask(layer(x=(1 << 20) + 8)) >= 7 * 32 * 2
    assert ask(layer(weight_pitch=33, weight_stride=600)) >= 3 * 16 * 32 * 2 and ask(layer(weight_stride=513)) >= 3 * 16 * 32 * 2
    assert ask(layer(), 1 << 22, 17) >= 7 * 16 * 2
    assert ask(layer(row_list=[0, 0, 0], x=None)) == 0
    assert lib.workers_dense_forward(None, None) == -1 and lib.workers_dense_workspace(C.byref(layer()), None, 0, None) == -1


@gpu
def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 16, device="cuda").bfloat16(), torch.zeros(2, 8, 16, device="cuda").bfloat16()
    for bad in (dict(rows=[4]), dict(rows=[3, 2]), dict(weight=w[:, :, :8]), dict(weight=w.half()), dict(weight_of=[0]), dict(activation="tanh"),
                dict(bias=torch.zeros(2, 9, device="cuda").bfloat16()), dict(y=torch.zeros(4, 8, device="cuda").half()), dict(x=x.cpu()), dict(x=x.T.contiguous().T),
                dict(residual=torch.zeros(4, 8, device="cuda")), dict(pre=torch.zeros(3, 8, device="cuda").bfloat16())):
        args = {**dict(x=x, weight=w, rows=[2, 2]), **bad}
        with pytest.raises((ValueError, ps.PSError)):
            workers_dense_forward(**args)
    with pytest.raises(TypeError):
        workers_dense_forward(x.double(), w.double(), [2, 2])
    with pytest.raises(ps.PSError):
        workers_dense_forward(x.float(), w.float(), [2, 2])
    with pytest.raises(ps.PSError):
        workers_dense_forward(x, w, [5, -1])
    dy = torch.zeros(4, 8, device="cuda").bfloat16()
    with pytest.raises(ValueError):
        workers_dense_backward(dy, x, w, [2, 2], dx_pre=torch.zeros_like(x))
    with pytest.raises(ValueError):
        workers_dense_backward(dy, x, w, [2, 2], dw=torch.zeros(2, 8, 16, device="cuda"), db=torch.zeros(2, 8, device="cuda").bfloat16())
