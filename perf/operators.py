"""The training operators for models of any shape: the AdamW step (over many tensors, and over the server's gradient queue) and the
workers' dense layer (forward and backward).  Each case is run either in plain elementary torch operations or, with `own` set,
through the framework's entry points.

    adamw      one AdamW step over many tensors at once, moments in 32 bits or in 8 (blocks of 256 with a power-of-two scale)
    queue      one server step with AdamW over a queue of gradients (the server's sync, replay and async modes)
    forward    y_g = act(x_g W_g^T + b_g) + r_g for workers g with ragged mini-batches, each on a weight snapshot of its own choice
    backward   dx = dy W + dx_add, dx_pre = dx * act'(x_pre), dW_g = dy_g^T x_g, db_g = the column sums of dy_g
"""
import math
import random

import numpy as np
import torch

own = False

PAPER_SIZES = (144, 16, 4608, 32, 802816, 512, 5120, 10)       # the paper's CNN: weights and biases in canonical order
PAPER_PARAMS, PAPER_STRIDE = 813258, 813312
BLOCK = 256                                                    # elements of a moment block in 8 bits
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the paper's CNN as eight tensors, everything in fp32: the smallest step, where latency counts
        dict(name="adamw paper model", op="adamw", layout="paper", total=PAPER_PARAMS, tensors=8, param="fp32", grad="fp32", copy="none",
             bits=32, clip=0.0, step=7),
        # mixed precision: fp32 weights, bf16 gradients and a bf16 copy that the layers read; odd sizes, clipped by global norm
        dict(name="adamw odd tensors, clipped", op="adamw", layout="odd", total=41000003, tensors=57, param="fp32", grad="bf16", copy="bf16",
             bits=32, clip=1.0, step=1200),
        # a model too large to keep its moments in 32 bits
        dict(name="adamw large, 8-bit moments", op="adamw", layout="model", total=400000000, tensors=61, param="fp32", grad="bf16", copy="bf16",
             bits=8, clip=0.0, step=3001),
        # one iteration of sixteen synchronous workers
        dict(name="queue sync 16", op="queue", mode="sync", K=16, tick=16, clip=0.0, step=3),
        # a deferred replay after an outage: 25 buffered ticks of 64 workers
        dict(name="queue replay 1600", op="queue", mode="replay", K=1600, tick=64, clip=0.0, step=40),
        # one update per arriving gradient
        dict(name="queue async 37", op="queue", mode="async", K=37, tick=37, clip=0.0, step=11),
        # answering one sample with the paper's dense layer: latency
        dict(name="forward one row", op="forward", type="bf16", groups=1, rows=1, spread="even", weights=1, K=1568, N=512, act="relu",
             bias=True, residual=False, pre=False, out="same"),
        # the paper's largest tick: 128 workers x 128 samples on a ring of 16 snapshots
        dict(name="forward 128 x 128", op="forward", type="bf16", groups=128, rows=16384, spread="even", weights=16, K=1568, N=512, act="relu",
             bias=True, residual=False, pre=True, out="same"),
        # a wide layer, ragged mini-batches, some workers with nothing to do
        dict(name="forward ragged", op="forward", type="fp16", groups=24, rows=9001, spread="ragged", weights=24, K=2048, N=5000, act="gelu",
             bias=True, residual=True, pre=True, out="same"),
        # decoding: a few rows for each of sixteen sets of weights, bound by reading them
        dict(name="forward few rows", op="forward", type="bf16", groups=16, rows=41, spread="ragged", weights=16, K=4096, N=4096, act="silu",
             bias=True, residual=True, pre=False, out="same"),
        # small workers on the paper's dense layer: gradients in fp32, one vector per worker
        dict(name="backward 16 x 64", op="backward", type="bf16", groups=16, rows=1024, spread="ragged", weights=4, K=1568, N=512, act="relu",
             add=False, raw=False, through=True, dw="fp32"),
        # one large batch through a square layer inside a residual block
        dict(name="backward large", op="backward", type="bf16", groups=1, rows=16384, spread="even", weights=1, K=4096, N=4096, act="gelu",
             add=True, raw=True, through=True, dw="same"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "queue", "forward", "forward", "backward", "backward"])
    if op == "adamw":
        param = rng.choice(["fp32", "fp32", "bf16"])
        return dict(op=op, layout=rng.choice(["odd", "odd", "model"]), total=_log(rng, 1500, 2.0e8), tensors=_log(rng, 1, 90), param=param,
                    grad=rng.choice(["fp32", "bf16", "fp16"]), copy=rng.choice(["none", "bf16", "fp16"]) if param == "fp32" else "none",
                    bits=rng.choice([32, 8]), clip=rng.choice([0.0, 0.5]), step=_log(rng, 1, 100000))
    if op == "queue":
        mode = rng.choice(["sync", "replay", "async"])
        tick = rng.randint(1, 64)
        K = tick * rng.randint(1, 12) if mode == "replay" else _log(rng, 1, 400)
        return dict(op=op, mode=mode, K=K, tick=tick if mode == "replay" else K, clip=rng.choice([0.0, 0.0, 0.5]), step=_log(rng, 1, 10000))
    groups = _log(rng, 1, 64)
    spread = rng.choice(["even", "ragged", "ragged"])
    K, N = _log(rng, 8, 8192), _log(rng, 8, 8192)
    most = 4.0e11 / (2.0 * K * N)
    rows = min(_log(rng, 1, 20000), max(1, int(most)))
    if rng.random() < 0.3:
        rows = min(rows, groups * rng.randint(1, 8))
    weights = rng.choice([1, groups, max(1, groups // 3)])
    weights = max(1, min(weights, int(3.0e8 / (K * N))))
    both = dict(op=op, type=rng.choice(["bf16", "fp16"]), groups=groups, rows=rows, spread=spread, weights=weights, K=K, N=N,
                act=rng.choice(["none", "relu", "gelu", "silu"]))
    if op == "forward":
        return dict(both, bias=rng.random() < 0.7, residual=rng.random() < 0.5, pre=rng.random() < 0.5, out=rng.choice(["same", "same", "fp32"]))
    groups = max(1, min(groups, int(1.0e9 / (K * N))))          # a gradient per worker
    return dict(both, groups=groups, weights=min(weights, groups), add=rng.random() < 0.3, raw=rng.random() < 0.5, through=rng.random() < 0.7,
                dw=rng.choice(["same", "fp32"]))


def tensor_sizes(case):
    if case["layout"] == "paper":
        return list(PAPER_SIZES)
    n, total = case["tensors"], case["total"]
    rng = random.Random(n * 1000003 + total)
    share = [math.exp(rng.uniform(0, 5)) for _ in range(n)] if case["layout"] == "odd" else [1.0 if i % 2 else 0.001 for i in range(n)]
    scale = total / sum(share)
    return [max(1, int(s * scale)) for s in share]


def group_rows(case):
    """Rows of each worker: equal, or uneven with some workers that have none."""
    G, M = case["groups"], case["rows"]
    if case["spread"] == "even":
        return [M // G + (1 if g < M % G else 0) for g in range(G)]
    rng = random.Random(G * 7919 + M)
    share = [0.0 if rng.random() < 0.1 else rng.expovariate(1.0) for _ in range(G)]
    if not sum(share):
        share[0] = 1.0
    edge = [0] + [round(M * sum(share[:g + 1]) / sum(share)) for g in range(G)]
    return [edge[g + 1] - edge[g] for g in range(G)]


def weight_of(case):
    return [g % case["weights"] for g in range(case["groups"])]


def work(case):
    size = {"fp32": 4, "bf16": 2, "fp16": 2, "none": 0}
    if case["op"] == "adamw":
        n = sum(tensor_sizes(case))
        per = 2 * size[case["param"]] + size[case["grad"]] + size[case["copy"]] + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)
        return {"bytes": int(per * n), "flops": 15 * n}
    if case["op"] == "queue":
        K = case["K"]
        updates = K if case["mode"] == "async" else 1
        return {"bytes": 4 * PAPER_PARAMS * (K + 6), "flops": PAPER_PARAMS * (K + 15 * updates)}
    rows = group_rows(case)
    M, K, N = sum(rows), case["K"], case["N"]
    used = len({w for w, r in zip(weight_of(case), rows) if r})
    if case["op"] == "forward":
        out = 4 if case["out"] == "fp32" else 2
        b = 2 * M * K + 2 * used * N * K + (2 * used * N if case["bias"] else 0) + M * N * (out + (2 if case["residual"] else 0) + (2 if case["pre"] else 0))
        return {"bytes": b, "flops": 2 * M * N * K}
    d = 4 if case["dw"] == "fp32" else 2
    b = 2 * M * N + 2 * M * K + 2 * used * N * K + case["groups"] * (N * K + N) * d
    b += 2 * M * K * ((1 if case["add"] else 0) + (1 if case["raw"] or not case["through"] else 0) + (2 if case["through"] else 0))
    return {"bytes": b, "flops": 4 * M * N * K}


# ---- inputs -----------------------------------------------------------------------------------------------------------
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
DECAY = 0.01
SEED = 0x5EED


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed * 7 + 1)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")                # noqa: E731
    s = {"case": case}
    if case["op"] == "adamw":
        sizes = tensor_sizes(case)
        at, n = [], 0
        for k in sizes:
            at.append(n)
            n += (k + BLOCK - 1) // BLOCK * BLOCK
        flat = lambda t: torch.zeros(n, dtype=t, device="cuda")                              # noqa: E731
        s.update(sizes=sizes, at=at, param=flat(TYPES[case["param"]]), grad=flat(TYPES[case["grad"]]),
                 copy=flat(TYPES[case["copy"]]) if case["copy"] != "none" else None)
        if case["bits"] == 32:
            s.update(m=flat(torch.float32), v=flat(torch.float32))
        else:
            s.update(m=flat(torch.uint8), v=flat(torch.uint8), m_scale=torch.zeros(n // BLOCK, dtype=torch.uint8, device="cuda"),
                     v_scale=torch.zeros(n // BLOCK, dtype=torch.uint8, device="cuda"))
        for i, (a, k) in enumerate(zip(at, sizes)):
            scale = 10.0 ** -(1 + i % 4)              # layers' gradients differ in magnitude
            s["param"][a:a + k] = normal(k) * 0.05
            g = normal(k) * scale
            s["grad"][a:a + k] = g
            m, v = g.roll(1) * 0.3 + normal(k) * 0.1 * scale, (g.roll(2) * 0.5).square() + 0.1 * scale * scale
            if case["bits"] == 32:
                s["m"][a:a + k], s["v"][a:a + k] = m, v
            else:
                end, b0, b1 = a + (k + BLOCK - 1) // BLOCK * BLOCK, a // BLOCK, (a + k + BLOCK - 1) // BLOCK
                pad = lambda t: torch.nn.functional.pad(t, (0, end - a - k)).view(-1, BLOCK)  # noqa: E731
                for name, value, kind in (("m", pad(m), "e4m3"), ("v", pad(v), "e5m2")):
                    codes, scales = _encode(value, kind, None)
                    s[name][a:end], s[name + "_scale"][b0:b1] = codes.view(-1), scales
        s["decay"] = [DECAY if k > 1000 else 0.0 for k in sizes]          # none on biases and norms
        if own:
            from paper_2406_05546_b200 import ps
            view = lambda t: [t[a:a + k] for a, k in zip(at, sizes)]                          # noqa: E731
            more = {}
            if case["bits"] == 8:
                blocks = lambda t: [t[a // BLOCK:(a + k + BLOCK - 1) // BLOCK] for a, k in zip(at, sizes)]   # noqa: E731
                more = dict(m_scale=blocks(s["m_scale"]), v_scale=blocks(s["v_scale"]))
            s["opt"] = ps.AdamW(view(s["param"]), view(s["grad"]), state_bits=case["bits"], weight_decay=s["decay"],
                                copies=view(s["copy"]) if s["copy"] is not None else None, m=view(s["m"]), v=view(s["v"]), **more)
        return s
    if case["op"] == "queue":
        K = case["K"]
        theta, m, v = normal(PAPER_STRIDE) * 0.05, normal(PAPER_STRIDE) * 0.003, normal(PAPER_STRIDE).square() * 1e-4
        for t in (theta, m, v):
            t[PAPER_PARAMS:] = 0
        s.update(m=m, v=v)
        if own:
            from paper_2406_05546_b200 import ps
            server = ps.ParameterServer(theta[:PAPER_PARAMS].cpu().numpy(), max_workers=1, max_batch=1, queue_slots=K)
            queue = torch.as_strided(server.slot_tensor(0), (K, PAPER_STRIDE), (PAPER_STRIDE, 1)) if K > 1 else server.slot_tensor(0).view(1, -1)
            s.update(server=server, ids=np.zeros(case["tick"], np.int32), bases=np.zeros(case["tick"], np.uint64),
                     mode={"sync": ps.SYNC, "replay": ps.REPLAY, "async": ps.ASYNC}[case["mode"]])
        else:
            queue = torch.empty(K, PAPER_STRIDE, device="cuda")
            s["theta"] = theta
        queue.normal_(0.0, 0.02, generator=gen)
        queue[:, PAPER_PARAMS:] = 0
        s["queue"] = queue
        return s
    rows, t = group_rows(case), TYPES[case["type"]]
    M, K, N = sum(rows), case["K"], case["N"]
    s.update(rows=rows, weight_of=weight_of(case), x=normal(M, K).to(t), weight=(normal(case["weights"], N, K) / math.sqrt(K)).to(t))
    if case["op"] == "forward":
        s["bias"] = normal(case["weights"], N).to(t) if case["bias"] else None
        s["residual"] = normal(M, N).to(t) if case["residual"] else None
        s["y"] = torch.empty(M, N, dtype=torch.float32 if case["out"] == "fp32" else t, device="cuda")
        s["pre"] = torch.empty(M, N, dtype=t, device="cuda") if case["pre"] else None
    else:
        d = torch.float32 if case["dw"] == "fp32" else t
        s["dy"] = (normal(M, N) * 0.1).to(t)
        s["x_pre"] = normal(M, K).to(t) if case["through"] else None
        s["dx_add"] = (normal(M, K) * 0.1).to(t) if case["add"] else None
        s["dx"] = torch.empty(M, K, dtype=t, device="cuda") if case["raw"] or not case["through"] else None
        s["dx_pre"] = torch.empty(M, K, dtype=t, device="cuda") if case["through"] else None
        s["dw"] = torch.empty(case["groups"], N, K, dtype=d, device="cuda")
        s["db"] = torch.empty(case["groups"], N, dtype=d, device="cuda")
    return s


# ---- the moments in 8 bits, in plain form ------------------------------------------------------------------------------
def _philox(counter, key):
    """Philox4x32-10 of int64 tensors that hold 32-bit words."""
    mask = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c0, c1, c2, c3


def _random16(n, tensor, step, seed):
    """Sixteen random bits per element: element i takes half word i % 8 of the generator's block i // 8."""
    j = torch.arange((n + 7) // 8, dtype=torch.int64, device="cuda")
    zero = torch.zeros_like(j)
    words = _philox((j & 0xFFFFFFFF, j >> 32, zero + tensor, zero + (step & 0xFFFFFFFF)), (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    w = torch.stack(words, 1)
    return torch.stack((w & 0xFFFF, w >> 16), 2).reshape(-1)


def _encode(x, kind, random16):
    """Blocks [n][256] of fp32 -> (codes, scales): code * 2^(scale - 127).  e4m3 to nearest even; e5m2 (values >= 0) by the random bits
    where given, a positive value never to zero.  What is not finite becomes the code for NaN and leaves the scale alone."""
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), torch.zeros_like(x)).amax(1)
    up = (most.view(torch.int32) + 0x1FFFFF) >> 23                   # exponent of the scale that puts the largest at 1.75 of the top binade at most
    scale = (up - (8 if kind == "e4m3" else 15)).clamp(1, 254)
    u = x * ((254 - scale) << 23).view(torch.float32)[:, None]
    if kind == "e4m3":
        code = torch.where(fine, u, torch.zeros_like(u)).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        r = (random16.view(x.shape) << 5).to(torch.int32) if random16 is not None else 1 << 20
        low = u < 2.0 ** -14
        bits = torch.where(low, u + 2.0 ** -14, torch.where(fine, u, torch.ones_like(u))).view(torch.int32) + r
        code = torch.where(low, (bits >> 21) - 113 * 4, (bits >> 21) - 112 * 4)
        code = torch.where((u > 0) & (code < 1), torch.ones_like(code), code).to(torch.uint8)
    return torch.where(fine, code, torch.full_like(code, 0x7F)), scale.to(torch.uint8)


def _decode(codes, scales, kind, t=torch.float32):
    value = codes.view(torch.float8_e4m3fn if kind == "e4m3" else torch.float8_e5m2).to(t).view(-1, BLOCK)
    return value * scales.view(torch.float8_e8m0fnu).to(t)[:, None]


# ---- the operators in plain form ---------------------------------------------------------------------------------------
def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _update(p, g, m, v, step, decay):
    """One AdamW update in fp32, every operation rounded by itself; returns the new (p, m, v)."""
    b1, b2, lr = HYPER["beta1"], HYPER["beta2"], HYPER["lr"]
    m = m * _f32(b1) + g * _f32(1.0 - b1)
    v = v * _f32(b2) + (g * _f32(1.0 - b2)) * g
    d = v.sqrt() * _f32(1.0 / math.sqrt(1.0 - b2 ** step)) + _f32(HYPER["eps"])
    return p * _f32(1.0 - lr * decay) - (m / d) * _f32(lr / (1.0 - b1 ** step)), m, v


def _plain_adamw(s):
    case = s["case"]
    factor = None
    if case["clip"]:
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for a, k in zip(s["at"], s["sizes"]):
            total += s["grad"][a:a + k].double().square().sum()
        factor = (case["clip"] / total.sqrt()).clamp(max=1.0).float()
    for i, (a, k) in enumerate(zip(s["at"], s["sizes"])):
        end = a + (k + BLOCK - 1) // BLOCK * BLOCK
        g = s["grad"][a:end].float()
        if factor is not None:
            g = g * factor
        if case["bits"] == 32:
            m, v = s["m"][a:end], s["v"][a:end]
        else:
            b = slice(a // BLOCK, end // BLOCK)
            m = _decode(s["m"][a:end], s["m_scale"][b], "e4m3").view(-1)
            v = _decode(s["v"][a:end], s["v_scale"][b], "e5m2").view(-1)
        p, m, v = _update(s["param"][a:end].float(), g, m, v, case["step"], s["decay"][i])
        s["param"][a:end] = p
        if s["copy"] is not None:
            s["copy"][a:end] = p
        if case["bits"] == 32:
            s["m"][a:end], s["v"][a:end] = m, v
        else:
            codes, s["m_scale"][b] = _encode(m.view(-1, BLOCK), "e4m3", None)
            s["m"][a:end] = codes.view(-1)
            codes, s["v_scale"][b] = _encode(v.view(-1, BLOCK), "e5m2", _random16(end - a, i, case["step"], SEED))
            s["v"][a:end] = codes.view(-1)


def _adamw_outputs(s):
    out = {"param": s["param"], "copy": s["copy"]}
    if s["case"]["bits"] == 32:
        return dict(out, m=s["m"], v=s["v"])
    # as the numbers they stand for: the codes times their blocks' scales
    return dict(out, m=s["m"].view(torch.float8_e4m3fn), v=s["v"].view(torch.float8_e5m2), m_scale=s["m_scale"].view(torch.float8_e8m0fnu),
                v_scale=s["v_scale"].view(torch.float8_e8m0fnu))


def _queue_factors(queue, case):
    """Each gradient's factor: the divisor of its mode, clipped by its own norm."""
    div = {"sync": case["K"], "replay": case["tick"], "async": 1}[case["mode"]]
    f = torch.full((queue.shape[0],), 1.0 / div, dtype=torch.float64, device="cuda")
    if case["clip"]:
        f = f * torch.stack([case["clip"] / q.double().norm() for q in queue]).clamp(max=1.0)
    return f


def _plain_queue(s):
    case, q = s["case"], s["queue"]
    f = _queue_factors(q, case).float()
    if case["mode"] == "async":
        for k in range(case["K"]):
            s["theta"], s["m"], s["v"] = _update(s["theta"], q[k] * f[k], s["m"], s["v"], case["step"] + k, DECAY)
    else:
        if case["clip"]:
            g = torch.zeros_like(s["theta"])
            for k0 in range(0, case["K"], 64):
                g = g + (q[k0:k0 + 64] * f[k0:k0 + 64, None]).sum(0)
        else:
            g = q.sum(0) * f[0]
        s["theta"], s["m"], s["v"] = _update(s["theta"], g, s["m"], s["v"], case["step"], DECAY)
    return {"theta": s["theta"], "m": s["m"], "v": s["v"]}


def _act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    return torch.ones_like(z)


def _groups(s):
    r0 = 0
    for g, (n, w) in enumerate(zip(s["rows"], s["weight_of"])):
        yield g, slice(r0, r0 + n), w
        r0 += n


def _plain_forward(s):
    case = s["case"]
    for _, r, w in _groups(s):
        z = s["x"][r].float() @ s["weight"][w].float().T
        if s["bias"] is not None:
            z = z + s["bias"][w].float()
        if s["pre"] is not None:
            s["pre"][r] = z
        y = _act(z, case["act"])
        s["y"][r] = y + s["residual"][r].float() if s["residual"] is not None else y
    return {"y": s["y"], "pre": s["pre"]}


def _plain_backward(s):
    case = s["case"]
    for g, r, w in _groups(s):
        dy = s["dy"][r].float()
        dx = dy @ s["weight"][w].float()
        if s["dx_add"] is not None:
            dx = dx + s["dx_add"][r].float()
        if s["dx"] is not None:
            s["dx"][r] = dx
        if s["dx_pre"] is not None:
            s["dx_pre"][r] = dx * _act_slope(s["x_pre"][r].float(), case["act"])
        s["dw"][g] = dy.T @ s["x"][r].float()
        s["db"][g] = dy.sum(0)
    return {k: s[k] for k in ("dx", "dx_pre", "dw", "db")}


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "adamw":
            _plain_adamw(s)
            return _adamw_outputs(s)
        return {"queue": _plain_queue, "forward": _plain_forward, "backward": _plain_backward}[case["op"]](s)
    from paper_2406_05546_b200 import ps
    if case["op"] == "adamw":
        s["opt"].ps_adamw_step(step=case["step"], clip_norm=case["clip"], seed=SEED, **HYPER)
        return _adamw_outputs(s)
    if case["op"] == "queue":
        server, tick = s["server"], case["tick"]
        for _ in range(case["K"] // tick):
            slots = server.ps_queue_reserve(tick)             # the workers' gradients are in their slots already
            server.ps_enqueue(s["ids"], s["bases"], 0, slot_ids=slots)
        server.ps_apply_adamw(s["mode"], s["m"], s["v"], step=case["step"], weight_decay=DECAY, clip_norm=case["clip"], **HYPER)
        return {"theta": server.head_tensor(), "m": s["m"], "v": s["v"]}
    if case["op"] == "forward":
        ps.workers_dense_forward(s["x"], s["weight"], s["rows"], weight_of=s["weight_of"], bias=s["bias"], residual=s["residual"],
                                 activation=case["act"], y=s["y"], pre=s["pre"])
        return {"y": s["y"], "pre": s["pre"]}
    ps.workers_dense_backward(s["dy"], s["x"], s["weight"], s["rows"], weight_of=s["weight_of"], x_pre=s["x_pre"], activation=case["act"],
                              dx_add=s["dx_add"], dx=s["dx"], dx_pre=s["dx_pre"], dw=s["dw"], db=s["db"])
    return {k: s[k] for k in ("dx", "dx_pre", "dw", "db")}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False                 # inputs only: no handle of the framework's
    try:
        s = prepare(case, seed)
    finally:
        own = was
    d = torch.float64
    lr, b1, b2, eps = HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"]

    def adamw(p, g, m, v, t, decay):
        m.mul_(b1).add_(g, alpha=1 - b1)
        v.mul_(b2).addcmul_(g, g, value=1 - b2)
        step = m / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt_() + eps)
        return p * (1 - lr * decay) - lr * step

    if case["op"] == "adamw":
        factor = 1.0
        if case["clip"]:
            norm = math.sqrt(sum(float(s["grad"][a:a + k].to(d).pow(2).sum()) for a, k in zip(s["at"], s["sizes"])))
            factor = min(1.0, case["clip"] / norm)
        out = {"param": torch.zeros(s["param"].shape, dtype=d, device="cuda")}
        narrow = case["bits"] == 8        # codes have no value in 64 bits: they are a rounding of the 32-bit moments
        if not narrow:
            out.update(m=torch.zeros_like(out["param"]), v=torch.zeros_like(out["param"]))
        for a, k, decay in zip(s["at"], s["sizes"], s["decay"]):
            if narrow:
                b = slice(a // BLOCK, (a + k + BLOCK - 1) // BLOCK)
                e = a + (k + BLOCK - 1) // BLOCK * BLOCK
                m = _decode(s["m"][a:e], s["m_scale"][b], "e4m3", d).view(-1)[:k]
                v = _decode(s["v"][a:e], s["v_scale"][b], "e5m2", d).view(-1)[:k]
            else:
                m, v = s["m"][a:a + k].to(d), s["v"][a:a + k].to(d)
            out["param"][a:a + k] = adamw(s["param"][a:a + k].to(d), s["grad"][a:a + k].to(d) * factor, m, v, case["step"], decay)
            if not narrow:
                out["m"][a:a + k], out["v"][a:a + k] = m, v
        out["copy"] = out["param"] if s["copy"] is not None else None
        return dict(out, m=None, v=None, m_scale=None, v_scale=None) if narrow else out
    if case["op"] == "queue":
        K = case["K"]
        div = {"sync": K, "replay": case["tick"], "async": 1}[case["mode"]]
        p, m, v = s["theta"].to(d), s["m"].to(d), s["v"].to(d)
        total = torch.zeros_like(p)
        for k in range(K):
            g = s["queue"][k].to(d)
            if case["clip"]:
                g = g * min(1.0, case["clip"] / float(torch.linalg.vector_norm(g)))
            if case["mode"] == "async":
                p = adamw(p, g, m, v, case["step"] + k, DECAY)
            else:
                total += g
        if case["mode"] != "async":
            p = adamw(p, total / div, m, v, case["step"], DECAY)
        return {"theta": p, "m": m, "v": v}
    edge = [0]
    for n in s["rows"]:
        edge.append(edge[-1] + n)
    zeros = lambda t: None if t is None else torch.zeros(t.shape, dtype=d, device="cuda")   # noqa: E731
    if case["op"] == "forward":
        out = {"y": zeros(s["y"]), "pre": zeros(s["pre"])}
        for g, w in enumerate(s["weight_of"]):
            lo, hi = edge[g], edge[g + 1]
            z = torch.einsum("mk,nk->mn", s["x"][lo:hi].to(d), s["weight"][w].to(d))
            if s["bias"] is not None:
                z += s["bias"][w].to(d)
            if out["pre"] is not None:
                out["pre"][lo:hi] = z
            if case["act"] == "relu":
                z = torch.where(z > 0, z, 0.0)
            elif case["act"] == "gelu":
                z = z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
            elif case["act"] == "silu":
                z = z * torch.sigmoid(z)
            out["y"][lo:hi] = z if s["residual"] is None else z + s["residual"][lo:hi].to(d)
        return out
    out = {k: zeros(s[k]) for k in ("dx", "dx_pre", "dw", "db")}
    for g, w in enumerate(s["weight_of"]):
        lo, hi = edge[g], edge[g + 1]
        dy = s["dy"][lo:hi].to(d)
        dx = torch.einsum("mn,nk->mk", dy, s["weight"][w].to(d))
        if s["dx_add"] is not None:
            dx += s["dx_add"][lo:hi].to(d)
        if out["dx"] is not None:
            out["dx"][lo:hi] = dx
        if out["dx_pre"] is not None:
            z = s["x_pre"][lo:hi].to(d)
            if case["act"] == "relu":
                dx = torch.where(z > 0, dx, 0.0)
            elif case["act"] == "gelu":
                dx = dx * (0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) * (2 * math.pi) ** -0.5)
            elif case["act"] == "silu":
                q = torch.sigmoid(z)
                dx = dx * (q + z * q * (1 - q))
            out["dx_pre"][lo:hi] = dx
        out["dw"][g] = torch.einsum("mn,mk->nk", dy, s["x"][lo:hi].to(d))
        out["db"][g] = torch.sum(dy, 0)
    return out
