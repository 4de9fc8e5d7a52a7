"""AdamW: the step over many tensors (32-bit and 8-bit moments) and the server step over the gradient queue, against the formula in float64 and,
for the 8-bit codes, against a bit-exact emulation of the documented rounding."""
import math

import numpy as np
import pytest
import torch

from paper_2406_05546_b200 import ps, synth
from paper_2406_05546_b200.ps import AdamW

gpu = pytest.mark.gpu
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8)
U = 2.0 ** -24            # largest relative error of one fp32 rounding
SIZES = [0, 1, 7, 255, 256, 257, 2047, 2048, 2049, 5003]


def formula(p, g, m, v, t, decay, lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8):
    """float64 update and the error bounds of its fp32 evaluation: every operation is off by U of its result, every constant by U.  m has two
    products and a sum of them, each term with a rounded constant: 3 U of the terms' sizes; v likewise with one product more: 4 U.  The step m / d: m's
    error, half v's (2 U), the root's 2^-23 (2 U), d's product and sum and two constants (4 U), the quotient's 2 ulp (4 U), its constant and product
    (2 U): 14 U; the weight: its own product and sum, with a rounded constant."""
    m_terms = beta1 * m.abs() + (1 - beta1) * g.abs()
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    d = (v / (1 - beta2 ** t)).sqrt() + eps
    size = lr / (1 - beta1 ** t)
    new = p * (1 - lr * decay) - size * m / d
    tiny = 2.0 ** -149     # the spacing of the smallest values
    e_m, e_v = 3 * U * m_terms + 2 * tiny, 4 * U * v + 2 * tiny
    e_p = 3 * U * p.abs() + U * new.abs() + size * (e_m + 14 * U * m.abs()) / d + tiny
    return new, m, v, e_p * 1.01, e_m * 1.01, e_v * 1.01


def flat(shape_list, make, offset=0, kind=torch.float32):
    """Views of one buffer with guard values between them."""
    views, n = [], 0
    places = []
    for k in shape_list:
        n = (n + 63) // 64 * 64 + 64 + offset
        places.append((n, k))
        n += k
    buf = torch.full((n + 64,), 77, dtype=kind, device="cuda")
    for a, k in places:
        buf[a:a + k] = make(k).to(kind)
        views.append(buf[a:a + k])
    mask = torch.ones(n + 64, dtype=torch.bool, device="cuda")
    for a, k in places:
        mask[a:a + k] = False
    return buf, views, mask


@gpu
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("kinds", [("fp32", "fp32", None), ("fp32", "bf16", "bf16"), ("fp32", "fp16", "fp16"), ("bf16", "bf16", None), ("fp16", "fp32", None)])
def test_many_tensors_against_the_formula(kinds, offset):
    kind = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
    tp, tg, tc = kind[kinds[0]], kind[kinds[1]], kind.get(kinds[2])
    gen = torch.Generator("cuda").manual_seed(3)
    normal = lambda s: lambda k: torch.randn(k, generator=gen, device="cuda") * s
    bufs = [flat(SIZES, normal(0.05), offset, tp), flat(SIZES, normal(0.02), offset, tg), flat(SIZES, normal(0.01), offset),
            flat(SIZES, lambda k: torch.rand(k, generator=gen, device="cuda") * 1e-3, offset)]
    copy = flat(SIZES, normal(1.0), offset, tc) if tc else None
    (pb, p, pm), (gb, g, _), (mb, m, mm), (vb, v, _) = bufs
    decay = [0.0 if k < 300 else 0.1 for k in SIZES]
    opt = AdamW(p, g, weight_decay=decay, copies=copy[1] if copy else None, m=m, v=v)
    for t in (1, 2, 900):
        before = [[x.double() for x in xs] for xs in (p, g, m, v)]
        opt.ps_adamw_step(step=t, **HYPER)
        torch.cuda.synchronize()
        for i, k in enumerate(SIZES):
            if k == 0:
                continue
            new, em, ev, e_p, e_m, e_v = formula(*(b[i] for b in before), t, decay[i])
            half = torch.finfo(tp).eps / 2 if tp != torch.float32 else 0.0
            small = torch.finfo(tp).smallest_normal * torch.finfo(tp).eps if half else 0.0
            assert ((p[i].double() - new).abs() <= e_p + half * (new.abs() + e_p) + small).all(), (t, k)
            assert ((m[i].double() - em).abs() <= e_m).all() and ((v[i].double() - ev).abs() <= e_v).all(), (t, k)
            if copy:
                assert torch.equal(copy[1][i], p[i].to(tc))
    for buf, _, mask in bufs[:1] + bufs[2:] + ([copy] if copy else []):
        assert (buf[mask] == 77).all()      # what lies between the tensors


@gpu
@pytest.mark.parametrize("state_bits", [32, 8])
@pytest.mark.parametrize("clip", [1e-3, 1e6])
def test_clipping_by_the_global_norm(clip, state_bits):
    gen = torch.Generator("cuda").manual_seed(5)
    p = [torch.randn(k, generator=gen, device="cuda") for k in (5, 70001, 1000)]
    g = [torch.randn(x.numel(), generator=gen, device="cuda").bfloat16() for x in p]
    q = [x.clone() for x in p]
    opt, ref = AdamW(p, g, state_bits=state_bits), AdamW(q, [x.float() for x in g], state_bits=state_bits)
    opt.ps_adamw_step(step=4, clip_norm=clip, grad_scale=0.5, **HYPER)
    norm = 0.5 * math.sqrt(sum(float(x.double().square().sum()) for x in g))
    factor = float(np.float32(0.5 * min(1.0, clip / norm)))
    info = opt.ps_adamw_read_info()
    assert info["grad_norm"] == pytest.approx(norm, rel=2 * U) and info["grad_factor"] == factor
    ref.ps_adamw_set_grads([x.float() * factor for x in g])
    ref.ps_adamw_step(step=4, **HYPER)
    for a, b in zip(p + opt.m + opt.v, q + ref.m + ref.v):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_gradient_that_is_not_finite(bad):
    p = [torch.ones(3000, device="cuda")]
    g = [torch.full((3000,), 0.5, device="cuda")]
    g[0][1234] = bad
    opt = AdamW(p, g)
    opt.ps_adamw_step(step=0, skip_nonfinite=True, **HYPER)
    assert opt.ps_adamw_read_info()["skipped_steps"] == 1 and opt.ps_adamw_read_info()["counted_steps"] == 0
    assert (p[0] == 1).all() and not opt.m[0].any() and not opt.v[0].any()
    opt.ps_adamw_step(step=0, **HYPER)
    fine = torch.ones(3000, dtype=torch.bool, device="cuda")
    fine[1234] = False
    assert torch.isfinite(p[0][fine]).all() and (p[0][fine] < 1).all() and torch.isnan(p[0][1234])
    g[0][1234] = 0.25
    opt.ps_adamw_step(step=0, skip_nonfinite=True, **HYPER)
    assert opt.ps_adamw_read_info() == pytest.approx({"counted_steps": 2, "skipped_steps": 1, "grad_norm": math.sqrt(2999 * 0.25 + 0.0625), "grad_factor": 1.0})


@gpu
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_a_gradient_that_is_not_finite(bad, bits):
    """An infinite norm makes the factor zero: every other element takes the step of a zero gradient.  A norm that is NaN reaches all of them."""
    gen = torch.Generator("cuda").manual_seed(4)
    p, q = ([torch.ones(k, device="cuda") for k in (3000, 77)] for _ in range(2))
    g = [torch.randn(k, generator=gen, device="cuda") for k in (3000, 77)]
    g[0][1234] = bad
    opt, ref = AdamW(p, g, state_bits=bits, weight_decay=0.1), AdamW(q, [torch.zeros_like(x) for x in g], state_bits=bits, weight_decay=0.1)
    for o in (opt, ref):
        o.ps_adamw_step(step=3, clip_norm=1.0, **HYPER)
    kind = (lambda xs: xs) if bits == 32 else (lambda xs: [x.view(torch.float8_e4m3fn).float() for x in xs])
    second = (lambda xs: xs) if bits == 32 else (lambda xs: [x.view(torch.float8_e5m2).float() for x in xs])
    for got, want in ((p, q), (kind(opt.m), kind(ref.m)), (second(opt.v), second(ref.v))):
        if math.isnan(bad):
            assert all(torch.isnan(x).all() for x in got)
        else:
            assert torch.isnan(got[0][1234])
            fine = torch.ones(3000, dtype=torch.bool, device="cuda")
            fine[1234] = False
            assert torch.equal(got[0][fine], want[0][fine]) and torch.equal(got[1], want[1])
    assert opt.ps_adamw_read_info()["grad_factor"] == pytest.approx(math.nan if math.isnan(bad) else 0.0, nan_ok=True)


@gpu
def test_a_captured_step_counts_and_follows_its_schedule():
    gen = torch.Generator("cuda").manual_seed(6)
    make = lambda: [torch.randn(k, generator=torch.Generator("cuda").manual_seed(k), device="cuda") for k in (300, 9001)]
    p, q, g = make(), make(), [torch.randn(k, generator=gen, device="cuda") for k in (300, 9001)]
    lr = torch.tensor([1e-3], device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        opt = AdamW(p, g, state_bits=8)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            opt.ps_adamw_step(lr=0.0, step=0, lr_dev=lr, seed=9, clip_norm=1.0)
    ref = AdamW(q, g, state_bits=8)
    for t in range(1, 5):
        lr.fill_(1e-3 / t)
        graph.replay()
        torch.cuda.synchronize()
        ref.ps_adamw_step(lr=float(np.float32(1e-3 / t)), step=t, seed=9, clip_norm=1.0)
        torch.cuda.synchronize()
        for a, b in zip(p + opt.m + opt.v + opt.m_scale + opt.v_scale, q + ref.m + ref.v + ref.m_scale + ref.v_scale):
            assert torch.equal(a, b), t
    assert opt.ps_adamw_read_info()["counted_steps"] == 4
    del graph


@gpu
@pytest.mark.parametrize("what", ["grads", "lr_dev"])
def test_replaced_tensors_stay_until_the_steps_that_read_them_are_done(what):
    """The optimizer works on a stream of its own, which is behind; what a step there reads is replaced and let go, and the other stream allocates anew."""
    n = 1 << 16
    side = torch.cuda.Stream()
    p, q = ([torch.ones(n, device="cuda")] for _ in range(2))
    grads, lr = [torch.full((n,), 0.5, device="cuda")], torch.full((n,), 1e-3, device="cuda")
    ref = AdamW(q, [grads[0].clone()])
    ref.ps_adamw_step(lr=0.0, step=1, lr_dev=lr.clone())
    opt, other_grads, other_lr = AdamW(p, grads, stream=side), [torch.full((n,), 3.0, device="cuda")], torch.zeros(n, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    opt.ps_adamw_step(lr=0.0, step=1, lr_dev=lr)
    if what == "grads":
        opt.ps_adamw_set_grads(other_grads)
    else:
        opt.ps_adamw_step(lr=0.0, step=2, lr_dev=other_lr)
    del grads, lr
    new = [torch.full((n,), -77.0, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    # (a step with learning rate 0 changes no weight)
    assert torch.equal(p[0], q[0]) and all((t == -77).all() for t in new)


@gpu
def test_gradients_that_are_refused_change_nothing():
    p, q = ([torch.ones(5000, device="cuda"), torch.ones(3, device="cuda")] for _ in range(2))
    grads, others = ([torch.full((k,), s, device="cuda") for k in (5000, 3)] for s in (0.5, -0.5))
    side = torch.cuda.Stream()
    opt, ref = AdamW(p, grads, stream=side), AdamW(q, grads)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(ps.PSError, match="PS_ERR_BAD_ARG"):
            opt.ps_adamw_set_grads(others)
        opt.ps_adamw_step(step=1, **HYPER)      # the capture goes on
    with pytest.raises(ValueError):
        opt.ps_adamw_set_grads(others[:1])
    with pytest.raises(ValueError):
        opt.ps_adamw_set_grads(others[::-1])
    graph.replay()
    torch.cuda.synchronize()
    opt.ps_adamw_step(step=2, **HYPER)
    for t in (1, 2):
        ref.ps_adamw_step(step=t, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p, q))
    del graph


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_a_list_without_elements_count(bits):
    empty = lambda: [torch.empty(0, device="cuda")]
    opt = AdamW(empty(), empty(), state_bits=bits)
    for more in (dict(step=0), dict(step=0, clip_norm=1.0), dict(step=0, skip_nonfinite=True), dict(step=5, clip_norm=1.0), dict(step=6)):
        opt.ps_adamw_step(**more, **HYPER)
    assert opt.ps_adamw_read_info() == {"counted_steps": 3, "skipped_steps": 0, "grad_norm": 0.0, "grad_factor": 1.0}


# ---- 8-bit moments, emulated ---------------------------------------------------------------------------------------------
def philox(counter, key):
    """Philox4x32-10 on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def half_words(n, tensor, step, seed):
    out = []
    for j in range((n + 7) // 8):
        for w in philox((j & 0xFFFFFFFF, j >> 32, tensor, step & 0xFFFFFFFF), (seed & 0xFFFFFFFF, seed >> 32)):
            out += [w & 0xFFFF, w >> 16]
    return np.array(out[:n], dtype=np.int64)


E4M3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()      # 0 .. 448, ascending
E5M2 = torch.arange(124, dtype=torch.uint8).view(torch.float8_e5m2).double().numpy()        # 0 .. 57,344


def scale_byte(x, most):
    """The smallest power of two that brings the largest finite value to `most` or below (floor 2^-126)."""
    x = np.abs(x[np.isfinite(x)])
    big = float(x.max()) if x.size else 0.0
    e = -126
    if big > 0:
        e = max(-126, math.ceil(math.log2(big / most)) - 2)
        while big > most * 2.0 ** e:
            e += 1
    return e


def quantize_m(x):
    codes, scales = np.zeros(len(x), np.uint8), []
    for b in range(0, len(x), 256):
        blk = x[b:b + 256].astype(np.float64)
        e = scale_byte(blk, 448.0)
        scales.append(e + 127)
        for i, val in enumerate(blk):
            if not np.isfinite(val):
                codes[b + i] = 0x7F
                continue
            u = abs(val) / 2.0 ** e
            hi = int(np.searchsorted(E4M3, u))
            lo = max(hi - 1, 0)
            if hi < len(E4M3):
                du, dl = E4M3[hi] - u, u - E4M3[lo]
                c = hi if du < dl or (du == dl and hi % 2 == 0) else lo
            else:
                c = lo
            codes[b + i] = c | (0x80 if np.signbit(val) else 0)
    return codes, np.array(scales)


def quantize_v(x, r):
    codes, scales = np.zeros(len(x), np.uint8), []
    for b in range(0, len(x), 256):
        blk = x[b:b + 256].astype(np.float64)
        e = scale_byte(blk, 57344.0)
        scales.append(e + 127)
        for i, val in enumerate(blk):
            if not np.isfinite(val):
                codes[b + i] = 0x7F
                continue
            u = np.float32(val / 2.0 ** e)
            if u < 2.0 ** -14:
                u = np.float32(u + np.float32(2.0 ** -14)) - np.float32(2.0 ** -14)      # what is left of it on the evenly spaced codes' grid
            lo = int(np.searchsorted(E5M2, u, side="right")) - 1
            if lo + 1 < len(E5M2):
                part = math.floor((float(u) - E5M2[lo]) / (E5M2[lo + 1] - E5M2[lo]) * 2 ** 21)
                lo += (part + (int(r[b + i]) << 5)) >> 21
            codes[b + i] = max(lo, 1) if val > 0 and np.float32(val / 2.0 ** e) > 0 else lo
    return codes, np.array(scales)


def fp32_update(p, g, m, v, t, decay, lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8):
    f = np.float32
    with np.errstate(all="ignore"):
        m = m * f(beta1) + g * f(1 - beta1)
        v = v * f(beta2) + (g * f(1 - beta2)) * g
        d = np.sqrt(v) * f(1 / math.sqrt(1 - beta2 ** t)) + f(eps)
        step = (m / d) * f(lr / (1 - beta1 ** t))
        return p * f(1 - lr * decay) - step, m, v, np.abs(step)


@gpu
@pytest.mark.parametrize("kind", ["ordinary", "wide", "zeros", "tiny", "huge", "not finite"])
@pytest.mark.parametrize("n", [1, 255, 257, 2500])
@pytest.mark.parametrize("offset", [0, 3])
def test_8_bit_moments_bit_for_bit(n, kind, offset):
    rng = np.random.default_rng(n + 10 * offset)
    shape = lambda: rng.standard_normal(n).astype(np.float32)
    scale = {"ordinary": 1e-2, "wide": 10.0 ** rng.uniform(-9, 2, n), "zeros": 0.0, "tiny": 1e-30, "huge": 1e17, "not finite": 1.0}[kind]
    pad = lambda a: torch.cat([torch.zeros(offset, dtype=a.dtype), a]).cuda()[offset:]
    blocks = (n + 255) // 256
    p0 = shape()
    bufs = dict(p=pad(torch.from_numpy(p0.copy())), g=pad(torch.zeros(n)), m=pad(torch.zeros(n, dtype=torch.uint8)), v=pad(torch.zeros(n, dtype=torch.uint8)))
    sm, sv = torch.zeros(blocks, dtype=torch.uint8, device="cuda"), torch.zeros(blocks, dtype=torch.uint8, device="cuda")
    other = torch.zeros(5, device="cuda")      # the tensor under test is the second of the list
    opt = AdamW([other, bufs["p"]], [other.clone(), bufs["g"]], state_bits=8, weight_decay=0.1,
                m=[torch.zeros(5, dtype=torch.uint8, device="cuda"), bufs["m"]], v=[torch.zeros(5, dtype=torch.uint8, device="cuda"), bufs["v"]],
                m_scale=[torch.zeros(1, dtype=torch.uint8, device="cuda"), sm], v_scale=[torch.zeros(1, dtype=torch.uint8, device="cuda"), sv])
    seed = 0x123456789ABCDEF0
    p, m, v = p0, np.zeros(n, np.float32), np.zeros(n, np.float32)
    for t in range(1, 4):
        with np.errstate(over="ignore"):
            g = (shape() * scale).astype(np.float32)
        if kind == "not finite":
            g[rng.integers(0, n)] = [np.inf, np.nan, -np.inf][t - 1]
        bufs["g"].copy_(torch.from_numpy(g))
        opt.ps_adamw_step(step=t, seed=seed, **HYPER)
        p, m, v, step = fp32_update(p, g, m, v, t, 0.1)
        cm, em = quantize_m(m)
        cv, ev = quantize_v(v, half_words(n, 1, t, seed))
        got = bufs["p"].cpu().numpy()      # two roundings of the weight on either side; a step 14 U off on one, 8 U on the other
        with np.errstate(all="ignore"):
            assert ((np.abs(got.astype(np.float64) - p) <= 4 * U * np.abs(p) + 24 * U * step) | (np.isnan(got) & np.isnan(p))).all()
        p = got
        assert np.array_equal(sm.cpu().numpy(), em) and np.array_equal(sv.cpu().numpy(), ev)
        got_m, got_v = bufs["m"].cpu().numpy(), bufs["v"].cpu().numpy()
        assert np.array_equal(np.where(got_m & 0x7F == 0x7F, 0x7F, got_m), cm)
        assert np.array_equal(got_v, cv)
        m = (torch.from_numpy(cm).view(torch.float8_e4m3fn).float().numpy() * np.repeat(2.0 ** (em - 127.0), 256)[:n]).astype(np.float32)
        v = (torch.from_numpy(cv).view(torch.float8_e5m2).float().numpy() * np.repeat(2.0 ** (ev - 127.0), 256)[:n]).astype(np.float32)


@gpu
def test_8_bit_second_moments_follow_in_the_mean():
    """With gradients that stop, v falls by beta2 a step: the mean of 2^20 elements after n steps is beta2^n of the first, within the noise of
    their rounding (independent; each step moves an element to a neighbouring code at most, 25 % away, with probability below 0.1 % / 14 %)."""
    n, steps = 1 << 20, 60
    p, g = [torch.zeros(n, device="cuda")], [torch.randn(n, generator=torch.Generator("cuda").manual_seed(1), device="cuda")]
    opt = AdamW(p, g, state_bits=8)
    opt.ps_adamw_step(step=1, seed=4, **HYPER)
    mean = lambda: float((opt.v[0].view(torch.float8_e5m2).double() * opt.v_scale[0].view(torch.float8_e8m0fnu).double().repeat_interleave(256)).sum())
    first = mean()
    g[0].zero_()
    for t in range(2, steps + 2):
        opt.ps_adamw_step(step=t, seed=4, **HYPER)
    # per element and step a variance of at most 0.25^2 * 0.001 / 0.14 of its square; E v^4 / (E v^2)^2 = 3 for the squares of normal values
    sigma = math.sqrt(steps * 0.0625 * 0.0072 * 3 / n)
    assert mean() / first == pytest.approx(0.999 ** steps, abs=6 * sigma)


@gpu
@pytest.mark.parametrize("state_bits", [8, 32])
def test_a_tensor_past_32_bits(state_bits):
    """2^31 elements and some: the last ones, and those around the 2^31st, as a small tensor of the same values has them (whose second moments'
    random bits, another matter, are looked at above)."""
    n, tail = (1 << 31) + 2048 + 77, 2048 + 77
    kind = torch.uint8 if state_bits == 8 else torch.float32
    p, g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-tail:] = torch.randn(tail, generator=torch.Generator("cuda").manual_seed(2), device="cuda").bfloat16()
    m, v = (torch.zeros(n, dtype=kind, device="cuda") for _ in range(2))
    q, h = p[-tail:].clone(), g[-tail:].clone()
    opt, ref = AdamW([p], [g], state_bits=state_bits, m=[m], v=[v]), AdamW([q], [h], state_bits=state_bits)
    for o in (opt, ref):
        o.ps_adamw_step(step=1, clip_norm=0.25, **HYPER)
    torch.cuda.synchronize()
    assert opt.ps_adamw_read_info()["grad_norm"] == ref.ps_adamw_read_info()["grad_norm"]
    assert torch.equal(p[-tail:], q) and torch.equal(m[-tail:], ref.m[0])
    assert (p[: 1 << 20] == p[0]).all() and not m[: 1 << 20].any() and not v[: 1 << 20].any()
    opt.close()


# ---- the gradient queue --------------------------------------------------------------------------------------------------
def server(K, **more):
    theta = synth.init_params(1)
    srv = ps.ParameterServer(theta, max_workers=1, max_batch=1, queue_slots=K, **more)
    gen = torch.Generator("cuda").manual_seed(K)
    rows = torch.randn(K, ps.P_PAD, generator=gen, device="cuda") * 0.03
    rows[:, ps.P:] = 0
    for k in range(K):
        srv.slot_tensor(k).copy_(rows[k])
    m = torch.randn(ps.P_PAD, generator=gen, device="cuda") * 0.01
    v = torch.rand(ps.P_PAD, generator=gen, device="cuda") * 1e-4
    return srv, torch.from_numpy(theta).cuda().double(), rows[:, :ps.P].double(), m, v


def enqueue(srv, K, tick, bases=None):
    for i in range(K // tick):
        slots = srv.ps_queue_reserve(tick)
        srv.ps_enqueue(list(range(tick)), bases if bases is not None else [0] * tick, i, slot_ids=slots)


def near(got, want, bound):
    assert ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() - bound).max())


@gpu
@pytest.mark.parametrize("K,tick,mode", [(1, 1, "SYNC"), (5, 5, "SYNC"), (161, 161, "SYNC"), (12, 4, "REPLAY"), (200, 8, "REPLAY")])
@pytest.mark.parametrize("clip", [0.0, 1.5])
def test_queue_summed(K, tick, mode, clip):
    srv, theta, rows, m, v = server(K, chain_len=2, ckpt_every=1)
    m0, v0 = m[:ps.P].double(), v[:ps.P].double()
    enqueue(srv, K, tick)
    res = srv.ps_apply_adamw(getattr(ps, mode), m, v, step=9, weight_decay=0.1, scale=0.5, clip_norm=clip, **HYPER)
    assert res == {"applied": K, "new_version": 1, "checkpointed": 1, "replicated": 1}
    f = torch.full((K,), 0.5 / (K if mode == "SYNC" else tick), dtype=torch.float64, device="cuda")
    if clip:
        f = f * (clip / rows.norm(dim=1)).clamp(max=1.0)
    terms = (rows.abs() * f[:, None]).sum(0)
    g = (rows * f[:, None]).sum(0)
    new, em, ev, e_p, e_m, e_v = formula(theta, g, m0, v0, 9, 0.1)
    # the sum: eight running sums of at most K / 8 terms each, joined in pairs, and up to sixteen ranges; factors and norms (of 2^20 squares,
    # summed in trees and runs of at most 50) are off by less than 40 U
    e_g = (K / 8 + 25 + (40 if clip else 0)) * U * terms
    d = (ev / (1 - 0.999 ** 9)).sqrt() + 1e-8
    # what an error of g does to m, v, and the step: dm = 0.1 e, dv = 2 * 0.001 |g| e
    e_m, e_v = e_m + 0.1 * e_g, e_v + 0.001 * (2 * g.abs() + e_g) * e_g
    size = 2e-3 / (1 - 0.9 ** 9)
    e_p = e_p + size * 0.1 * e_g / d + size * em.abs() / d * (0.001 * (2 * g.abs() + e_g) * e_g / ev)
    head = srv.head_tensor()
    near(head[:ps.P], new, e_p)
    near(m[:ps.P], em, e_m)
    near(v[:ps.P], ev, e_v)
    assert not head[ps.P:].any() and not m[ps.P:].any() and not v[ps.P:].any()
    for which in (-1, 1000):
        assert np.array_equal(srv.ps_export_params(which)[0], head[:ps.P].cpu().numpy())
    assert srv.ps_stats()["queue_len"] == 0
    srv.close()


@gpu
@pytest.mark.parametrize("K", [1, 9, 300])
@pytest.mark.parametrize("treated", [False, True])
def test_queue_in_order(K, treated):
    srv, theta, rows, m, v = server(K, ring_depth=3, chain_len=2, replicate_every=2)
    p, em, ev = (t[:ps.P].cpu().numpy() for t in (srv.head_tensor(), m, v))
    order = np.random.default_rng(2).permutation(K).astype(np.int32)
    enqueue(srv, K, K)
    more = dict(clip_norm=2.0, staleness_alpha=0.5) if treated else {}
    srv.ps_apply_adamw(ps.ASYNC, m, v, step=2, weight_decay=0.1, scale=0.5, order=order, **more, **HYPER)
    g32 = rows.float().cpu().numpy()
    norms = rows.norm(dim=1).cpu().numpy()
    versions, bound = [], 0.0
    for j, k in enumerate(order):
        f = np.float32(0.5 / (1.0 + 0.5 * j)) * np.float32(min(1.0, 2.0 / norms[k])) if treated else np.float32(0.5)
        p, em, ev, step = fp32_update(p, np.float32(f) * g32[k], em, ev, 2 + j, 0.1)
        versions = (versions + [p])[-3:]
        bound = bound + 4 * U * np.abs(p) + 24 * U * step      # as for one update
    head = srv.head_tensor()[:ps.P].cpu().numpy()
    if treated:      # the factor is off by 64 U at most (a norm of 2^20 squares in runs of 50), and m and v with it: twice as much of a step's length
        assert np.abs(head - p).max() <= bound.max() + K * 128 * U * 2e-3
    else:
        assert (np.abs(head - p) <= bound).all() and np.array_equal(m[:ps.P].cpu().numpy(), em) and np.array_equal(v[:ps.P].cpu().numpy(), ev)
        for lag in range(min(K, 3)):
            off = srv.ps_pull_snapshot(0, lag).dev_ptr - srv.arena.data_ptr()
            assert (np.abs(srv.arena[off:off + ps.P * 4].view(torch.float32).cpu().numpy() - versions[-1 - lag]) <= bound).all()
        if K == 9:       # version 8 is the latest replication event
            off = srv.ps_pull_snapshot(0, 1).dev_ptr - srv.arena.data_ptr()
            assert np.array_equal(srv.ps_export_params(-1)[0], srv.arena[off:off + ps.P * 4].view(torch.float32).cpu().numpy())
    srv.close()


@gpu
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("mode", ["SYNC", "REPLAY", "ASYNC"])
def test_queue_clipping_a_gradient_that_is_not_finite(bad, mode):
    """Its factor is zero where its norm is infinite, as if the gradient were zero elsewhere, and NaN where it is NaN.  What SGD makes of it is unchanged:
    a norm that is NaN clips nothing."""
    where, fine = 5000, torch.arange(ps.P_PAD, device="cuda") < ps.P
    results = []
    for value in (bad, 0.0):
        srv, _, _, m, v = server(3)
        if value == 0.0:
            srv.slot_tensor(1).zero_()
        else:
            srv.slot_tensor(1)[where] = value
        enqueue(srv, 3, 3)
        srv.ps_apply_adamw(getattr(ps, mode), m, v, step=2, clip_norm=0.5, **HYPER)
        results.append((srv.head_tensor().clone(), m, v))
        srv.close()
    for got, want in zip(*results):
        assert not got[ps.P:].any()
        if math.isnan(bad):
            assert torch.isnan(got[:ps.P]).all()
        else:
            assert torch.isnan(got[where])
            fine[where] = False
            assert torch.equal(got[fine], want[fine])
    if math.isnan(bad):
        srv, theta, rows, _, _ = server(1)
        srv.slot_tensor(0)[where] = bad
        enqueue(srv, 1, 1)
        srv.ps_apply_stale(getattr(ps, mode), 1.0, clip_norm=0.5)
        new = srv.head_tensor()[:ps.P].double()
        fine = fine[:ps.P]
        fine[where] = False
        assert torch.isnan(new[where]) and ((new - (theta - rows[0])).abs() <= U * (theta - rows[0]).abs() * 1.01)[fine].all()
        srv.close()


@gpu
@pytest.mark.parametrize("mode", ["SYNC", "ASYNC"])
def test_queue_clipping_to_less_than_fp32_holds(mode):
    """A clip_norm below the smallest fp32 value clips to nothing; it does not switch clipping off."""
    results = []
    for clip in (1e-60, 0.0):
        srv, _, _, m, v = server(3)
        if clip == 0.0:
            srv.slot_tensor(0).view(1, -1).as_strided((3, ps.P_PAD), (ps.P_PAD, 1)).zero_()
        enqueue(srv, 3, 3)
        srv.ps_apply_adamw(getattr(ps, mode), m, v, step=2, clip_norm=clip, **HYPER)
        results.append((srv.head_tensor().clone(), m, v))
        srv.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))


@gpu
@pytest.mark.parametrize("rows", [[64, 9, 0, 130], [16] * 6])
@pytest.mark.parametrize("mode", ["SYNC", "ASYNC"])
def test_the_dense_layer_writes_where_the_servers_step_reads(rows, mode):
    """The CNN's dense layer, 1568 -> 512, on the workers' own batches: its weight and bias gradients go straight into the workers' rows of the gradient queue,
    beside what other layers have put there, and the server's step takes them from there; the next forward call reads the new weights."""
    F1W, F1B, K, N, G = 4800, 807616, 1568, 512, len(rows)
    srv, theta, other, m, v = server(G)
    gen = torch.Generator("cuda").manual_seed(3)
    M = sum(rows)
    x, dy = torch.randn(M, K, generator=gen, device="cuda").bfloat16(), (torch.randn(M, N, generator=gen, device="cuda") * 0.02).bfloat16()
    layer = lambda: srv.head_tensor()[F1W:F1W + N * K].view(1, N, K).bfloat16()
    queue = torch.as_strided(srv.slot_tensor(0), (G, ps.P_PAD), (ps.P_PAD, 1))
    at = lambda first, shape, strides: torch.as_strided(queue, shape, strides, queue.storage_offset() + first)
    ps.workers_dense_backward(dy, x, layer(), rows, [0] * G, dw=at(F1W, (G, N, K), (ps.P_PAD, K, 1)), db=at(F1B, (G, N), (ps.P_PAD, 1)))
    ps.workers_dense_status()
    grads = queue[:, :ps.P].double()
    first = 0
    for g, n in enumerate(rows):
        gx, gy = x[first:first + n].double(), dy[first:first + n].double()
        first += n
        want = other[g].clone()
        want[F1W:F1W + N * K], want[F1B:F1B + N] = (gy.T @ gx).view(-1), gy.sum(0)
        bound = torch.zeros_like(want)      # an accumulator drops less than 2^-22 of its terms a time, sixteen products each; the result is rounded once
        bound[F1W:F1W + N * K], bound[F1B:F1B + N] = (gy.abs().T @ gx.abs()).view(-1), gy.abs().sum(0)
        near(queue[g, :ps.P], want, bound * (n / 16 + 2) * 2.0 ** -22 + (bound > 0) * want.abs() * 2.0 ** -23)
    assert not queue[:, ps.P:].any()
    m0, v0 = m[:ps.P].cpu().numpy(), v[:ps.P].cpu().numpy()
    enqueue(srv, G, G)
    srv.ps_apply_adamw(getattr(ps, mode), m, v, step=3, weight_decay=0.1, **HYPER)
    head = srv.head_tensor()[:ps.P]
    if mode == "ASYNC":
        p = theta.float().cpu().numpy()
        bound = 0.0
        for j in range(G):
            p, m0, v0, step = fp32_update(p, grads[j].float().cpu().numpy(), m0, v0, 3 + j, 0.1)
            bound = bound + 4 * U * np.abs(p) + 24 * U * step      # as in test_queue_in_order
        assert (np.abs(head.cpu().numpy() - p) <= bound).all()
    else:
        new, em, ev, e_p, _, _ = formula(theta, grads.mean(0), torch.from_numpy(m0).cuda().double(), torch.from_numpy(v0).cuda().double(), 3, 0.1)
        e_g, d = (G / 8 + 25) * U * grads.abs().mean(0), (ev / (1 - 0.999 ** 3)).sqrt() + 1e-8      # as in test_queue_summed
        near(head, new, e_p + 2e-3 / (1 - 0.9 ** 3) * (0.1 * e_g / d + em.abs() / d * (0.001 * (2 * grads.mean(0).abs() + e_g) * e_g / ev)))
    w = layer()
    y = ps.workers_dense_forward(x, w, rows, [0] * G, out_dtype=torch.float32)
    terms = x.double().abs() @ w[0].double().abs().T
    assert torch.equal(w[0].view(-1), head[F1W:F1W + N * K].bfloat16())
    near(y, x.double() @ w[0].double().T, terms * (32 + K / 512 + 12) * 2.0 ** -22)
    srv.close()


@gpu
def test_queue_padding_stays_zero():
    srv, theta, rows, m, v = server(3)
    m[ps.P:], v[ps.P:] = 1.0, 1.0
    enqueue(srv, 3, 3)
    srv.ps_apply_adamw(ps.ASYNC, m, v, **HYPER)
    assert not srv.head_tensor()[ps.P:].any() and not m[ps.P:].any() and not v[ps.P:].any()
    srv.close()


@gpu
def test_refusals():
    p, g = [torch.ones(10, device="cuda")], [torch.ones(10, device="cuda")]
    opt = AdamW(p, g)
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-60), dict(lr=math.nan), dict(step=-1), dict(clip_norm=-1.0),
                dict(clip_norm=math.nan), dict(grad_scale=math.inf)):
        with pytest.raises(ps.PSError, match="PS_ERR_BAD_ARG"):
            opt.ps_adamw_step(**{**HYPER, "step": 1, **bad})
    assert (p[0] == 1).all()
    with pytest.raises(ValueError):
        AdamW(p, [torch.ones(11, device="cuda")])
    with pytest.raises(ValueError):
        AdamW(p, [torch.ones(20, device="cuda")[::2]])
    with pytest.raises(ValueError):
        AdamW(p, g, m_scale=[torch.zeros(1, dtype=torch.uint8, device="cuda")])
    with pytest.raises(ps.PSError):
        AdamW([x.bfloat16() for x in p], g, copies=[x.bfloat16() for x in p])
    with pytest.raises(ps.PSError):
        AdamW(p, g, weight_decay=-1.0)
    with pytest.raises(ps.PSError):
        AdamW(p, g, state_bits=16)
    srv, _, _, m, v = server(2)
    enqueue(srv, 2, 2)
    for bad in (dict(step=0), dict(weight_decay=-0.1), dict(staleness_alpha=-1.0), dict(eps=0.0), dict(clip_norm=-1.0)):
        with pytest.raises(ps.PSError, match="PS_ERR_BAD_ARG"):
            srv.ps_apply_adamw(ps.SYNC, m, v, **{**HYPER, **bad})
    with pytest.raises(ps.PSError, match="PS_ERR_BAD_ARG"):
        srv.ps_apply_adamw(ps.SYNC, m, m, **HYPER)
    assert srv.ps_stats()["queue_len"] == 2 and srv.ps_stats()["version"] == 0
    srv.close()


@gpu
def test_queue_moments_that_share_memory_are_refused():
    srv, _, _, _, _ = server(2)
    enqueue(srv, 2, 2)
    both = torch.zeros(ps.P_PAD + 4, device="cuda")
    for one, other in ((both[:-4], both[4:]), (both[4:], both[:-4])):
        with pytest.raises(ps.PSError, match="PS_ERR_BAD_ARG"):
            srv.ps_apply_adamw(ps.SYNC, one, other, **HYPER)
    assert srv.ps_stats()["queue_len"] == 2 and srv.ps_stats()["version"] == 0
    srv.close()


# ---- without a GPU -------------------------------------------------------------------------------------------------------
def test_shared_memory_is_refused():
    """A tensor given twice, or moments that two share, would be stepped by two pieces at once.  (Nothing is launched: the addresses are never read.)"""
    import ctypes as C
    lib = ps.load()

    def create(*places, bits=32):
        """places: (n, param, copy, m, v, m_scale, v_scale)"""
        cfg, t, opt = ps.AdamWConfig(), (ps.AdamWTensor * len(places))(), C.c_void_p()
        cfg.state_bits, cfg.copy_type = bits, ps.TYPE_BF16
        for a, (n, p, c, m, v, ms, vs) in zip(t, places):
            a.n, a.param, a.grad, a.copy, a.m, a.v, a.m_scale, a.v_scale = n, p, 1 << 30, c, m, v, ms, vs
        rc = lib.ps_adamw_create(C.byref(cfg), t, len(places), C.byref(opt))      # no arena: refused in any case, with a message of its own
        text = lib.ps_last_error(None).decode()
        assert rc == -1 and ("share memory" in text) != ("arena" in text)
        return "share memory" in text
    K = 1 << 20
    one, two = (100, K, None, 2 * K, 3 * K, None, None), (100, 4 * K, None, 5 * K, 6 * K, None, None)
    assert not create(one) and not create(one, two) and not create(one, (100, K + 400, None, 2 * K + 400, 3 * K + 400, None, None))
    assert create(one, one) and create(one, two, (100, K + 396, None, 7 * K, 8 * K, None, None))
    assert create((100, K, None, 2 * K, 2 * K, None, None)) and create((100, K, None, K, 2 * K, None, None)) and create((100, K, K, 2 * K, 3 * K, None, None))
    assert create(one, (100, 4 * K, None, 2 * K, 6 * K, None, None)) and create(one, (100, 4 * K, None, 5 * K, 3 * K, None, None))
    assert not create(one, (0, K, None, 2 * K, 3 * K, None, None))
    small = (257, K, None, 2 * K, 3 * K, 4 * K, 5 * K)
    assert not create(small, bits=8) and create((257, K, None, 2 * K, 2 * K + 256, 4 * K, 5 * K), bits=8) and create((257, K, None, 2 * K, 3 * K, 4 * K, 4 * K + 1), bits=8)
    assert not create((257, K, None, 2 * K, 3 * K, 4 * K, 4 * K + 2), bits=8)


def test_query_bytes_checks_its_arguments():
    import ctypes as C
    lib = ps.load()
    cfg, t, size = ps.AdamWConfig(), (ps.AdamWTensor * 2)(), C.c_uint64()
    cfg.state_bits, cfg.param_type, cfg.grad_type = 32, ps.TYPE_FP32, ps.TYPE_BF16
    t[0].n, t[1].n = 5000, 0
    ask = lambda n=2: lib.ps_adamw_query_bytes(C.byref(cfg), t, n, C.byref(size))
    assert ask() == 0 and 0 < size.value < 1 << 20
    assert ask(0) == -1 and ask(-3) == -1
    for field, bad in (("state_bits", 16), ("param_type", 3), ("grad_type", -1)):
        good = getattr(cfg, field)
        setattr(cfg, field, bad)
        assert ask() == -1
        setattr(cfg, field, good)
    t[1].n = -1
    assert ask() == -1
    t[1].n, t[0].weight_decay = 0, math.nan
    assert ask() == -1
    assert lib.ps_adamw_query_bytes(None, t, 2, C.byref(size)) == -1 and lib.ps_adamw_create(None, None, 1, None) == -1
    assert lib.ps_adamw_step(None, None) == -1 and lib.ps_adamw_destroy(None) == -1 and lib.ps_adamw_set_grads(None, None) == -1
