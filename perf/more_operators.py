"""Feed-forward blocks of packed matrices, and their products with 8-bit tokens, as measurable cases.

Five operators.  `tokens8`: tokens to 8-bit integers with a scale each.  `project8`: such tokens through one packed matrix, whose scales
are a channel's within each chunk.  `gated8`: such tokens through two packed matrices, act(gate) * up.  `gated`: the same of unrounded tokens, as a
training step has it, with what its way back needs.  `gated_grad`: that way back.  Shapes are those of the benchmark's
decoder blocks and generic ones of the same ranges.

A case holds: op; rows, cols, G (chunk width), unit_rows (0 = whole columns), tokens, plan ("policy": the trained policy's mix at about 2 bits, "even": all
seven treatments alike), dtype (of the tokens, of what comes out, and of the weights that stay as they are), act ("silu", "gelu", "gelu_tanh"), and save
(gated alone: both products are written too).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
POLICY = (0.0866 / 4, 0.0866 / 4, 0.0866 / 4, 0.0866 / 4, 0.1565, 0.3654, 0.3915)
LEVELS = (0, 255, 15, 7, 3, 0, 0)                # largest code of the uniform treatments


def _case(name, op, rows, cols, tokens, G=128, unit_rows=0, dtype="bf16", plan="policy", act="silu", save=False):
    c = dict(op=op, rows=rows, cols=cols, tokens=tokens, G=G, unit_rows=unit_rows, dtype=dtype, plan=plan, act=act, save=save)
    return dict(c, name=name) if name else c


def listed():
    return [
        # what a prompt of 4096 tokens hands to a 7B block's down projection
        _case("tokens8_4096_7b", "tokens8", 0, 11008, 4096),
        # a decoding step of seven requests in a small fp32 layer: latency
        _case("tokens8_7_f32", "tokens8", 0, 1056, 7, G=96, dtype="f32"),
        # one token through a 7B block's attention projection: latency
        _case("project8_1_attn_7b", "project8", 4096, 4096, 1),
        # a decoding step of 48 requests through a 7B block's up projection
        _case("project8_48_up_7b", "project8", 11008, 4096, 48),
        # a prompt of 2000 tokens through a 7B block's down projection
        _case("project8_2000_down_7b", "project8", 4096, 11008, 2000),
        # a small layer of odd sizes with every treatment, fp32 results
        _case("project8_ragged_f32", "project8", 1000, 1056, 77, G=96, dtype="f32", plan="even"),
        # a decoding step of 16 requests through a 7B block's gate and up projections
        _case("gated8_16_7b", "gated8", 11008, 4096, 16),
        # a prompt of 1024 tokens through those of a 13B block in tile units
        _case("gated8_1024_13b", "gated8", 13824, 5120, 1024, unit_rows=128),
        # one token through a 7B block's gate and up projections, tokens as they are
        _case("gated_1_7b", "gated", 11008, 4096, 1),
        # the forward pass of a training step over the same, with what the way back needs
        _case("gated_2048_7b", "gated", 11008, 4096, 2048, save=True),
        # its way back
        _case("gated_grad_2048_7b", "gated_grad", 11008, 4096, 2048),
        # a small fp32 layer of odd sizes, every treatment, on its way back
        _case("gated_grad_ragged_f32", "gated_grad", 1000, 1056, 77, G=96, dtype="f32", plan="even", act="gelu_tanh"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tokens8", "project8", "project8", "gated8", "gated", "gated_grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    G = rng.choice([64, 64, 96, 128, 128, 128, 256])
    cols = G * _log(rng, 4, 11008 // G)
    if op == "tokens8":
        return _case(None, op, 0, cols, _log(rng, 1, min(8192, 40_000_000 // cols)), G, dtype=dtype)
    unit_rows = rng.choice([0, 0, 0, 128])
    tokens = _log(rng, 1, 2048)
    pair = op != "project8"
    most = (11008 * 4096 if pair else 13824 * 5120) if dtype == "bf16" or not pair else 1 << 22
    rows = 8 * _log(rng, 32, max(33, min(13824, most // cols) // 8))
    if unit_rows:
        rows = max(unit_rows, rows // unit_rows * unit_rows)
    if dtype == "f32":
        tokens = min(tokens, 1024)
    return _case(None, op, rows, cols, tokens, G, unit_rows, dtype, rng.choice(["policy", "policy", "even"]),
                 rng.choice(["silu", "silu", "gelu", "gelu_tanh"]) if pair else "silu", op == "gated" and rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _type(word):
    return torch.float32 if word == "f32" else torch.bfloat16


def _bytes_per_group(a, G):
    return (G + 4) // 5 if a == 5 else {0: 0, 1: G, 2: G // 2, 3: G * 3 // 8, 4: G // 4, 6: G // 8}[a]


def _plan(case, rng):
    """(action per unit, offset of each unit's codes, rows of a unit), as a controller leaves them."""
    R_u = case["unit_rows"] or case["rows"]
    U = case["rows"] // R_u * (case["cols"] // case["G"])
    action = rng.choice(7, size=U, p=np.array(POLICY) if case["plan"] == "policy" else np.full(7, 1 / 7))
    payload = np.array([(_bytes_per_group(a, case["G"]) * R_u + 15) // 16 * 16 for a in range(7)])[action]
    return action.astype(np.uint8), np.concatenate([[0], np.cumsum(payload)]).astype(np.int64), R_u


def _pack(w, a, codes, base, scale, offset, groups):
    """Fits and packs the units w [units, R_u, G] at treatment a, each at its place of the code stream."""
    G = w.shape[2]
    if a == 5 or a == 6:
        size = w.abs().mean(2)
        offset[groups] = 0.0
        scale[groups] = size
        q = (w >= 0) if a == 6 else torch.clamp(torch.round(w / size[:, :, None]), -1, 1) + 1
    else:
        lo = 0.9 * w.amin(2)
        step = (0.9 * w.amax(2) - lo) / LEVELS[a]
        offset[groups] = lo
        scale[groups] = step
        q = torch.clamp(torch.round((w - lo[:, :, None]) / step[:, :, None]), 0, LEVELS[a])
    q = q.to(torch.int32)
    if a == 5:
        q = torch.nn.functional.pad(q, (0, -G % 5)).reshape(*q.shape[:2], -1, 5)
        data = (q * torch.tensor([1, 3, 9, 27, 81], dtype=torch.int32, device=DEV)).sum(3)
    else:
        b = {1: 8, 2: 4, 3: 3, 4: 2, 6: 1}[a]
        bits = (q[..., None] >> torch.arange(b, dtype=torch.int32, device=DEV)) & 1
        bits = bits.reshape(*q.shape[:2], -1, 8)
        data = (bits << torch.arange(8, dtype=torch.int32, device=DEV)).sum(3)
    data = data.reshape(w.shape[0], -1).to(torch.uint8)
    codes[base[:, None] + torch.arange(data.shape[1], device=DEV)] = data


def _packed_matrix(case, g, rng):
    """A matrix with a few large columns, and what packing it left: W, action, code_off, codes, scale, offset."""
    rows, cols, G = case["rows"], case["cols"], case["G"]
    W = 0.02 * torch.randn(rows, cols, generator=g, device=DEV)
    W[:, torch.randperm(cols, generator=g, device=DEV)[:max(1, cols // 100)]] *= 5.0
    W = W.to(_type(case["dtype"]))
    action, off, R_u = _plan(case, rng)
    U, nc = len(action), cols // G
    units = W.float().reshape(rows // R_u, R_u, nc, G).permute(0, 2, 1, 3).reshape(U, R_u, G)
    codes = torch.zeros(max(16, int(off[-1])), dtype=torch.uint8, device=DEV)
    scale = torch.zeros(U, R_u, device=DEV)
    offset = torch.zeros(U, R_u, device=DEV)
    for a in range(1, 7):
        at = torch.from_numpy(np.flatnonzero(action == a)).to(DEV)
        if len(at) == 0:
            continue
        for part in at.split(max(1, (1 << 23) // (R_u * G))):
            _pack(units[part], a, codes, torch.from_numpy(off).to(DEV)[part], scale, offset, part)
    return dict(W=W, action=torch.from_numpy(action).to(DEV), code_off=torch.from_numpy(off).to(DEV), codes=codes,
                scale=scale.reshape(-1), offset=offset.reshape(-1), R_u=R_u)


def _block(G):
    """Columns whose sum goes with a token: a chunk's, in parts of 128 at most."""
    steps = (G + 31) // 32
    parts = (steps + 3) // 4
    return 32 * ((steps + parts - 1) // parts)


def _eight(x, G):
    """x [T, cols] in 32 bits as (integers -127 .. 127, a scale a token, sums of the integers over blocks of columns, padded to fours)."""
    largest = x.abs().amax(1)
    sigma = largest / torch.full_like(largest, 127.0)
    q = torch.clamp(torch.round(x * (1.0 / sigma)[:, None]), -127, 127).to(torch.int8)
    sums = q.reshape(x.shape[0], -1, _block(G)).sum(2, dtype=torch.int32)
    return q, sigma, torch.nn.functional.pad(sums, (0, -sums.shape[1] % 4))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    T, cols, dtype, op = case["tokens"], case["cols"], _type(case["dtype"]), case["op"]
    s = dict(case=case)
    if op != "tokens8":
        s["plans"] = [_packed_matrix(case, g, rng) for _ in range(1 if op == "project8" else 2)]
    if op == "gated_grad":
        s["dH"] = (1e-3 * torch.randn(T, case["rows"], generator=g, device=DEV)).to(dtype)
        s["G"], s["U"] = ((1.7 * torch.randn(T, case["rows"], generator=g, device=DEV)).to(dtype) for _ in range(2))
        return s
    channel = torch.exp(0.5 * torch.randn(cols, generator=g, device=DEV))          # activations with channels of their own size
    s["X"] = (torch.randn(T, cols, generator=g, device=DEV) * channel).to(dtype)
    if op in ("project8", "gated8"):
        s["q"], s["sigma"], s["sums"] = _eight(s["X"].float(), case["G"])           # several projections take the same tokens
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _dequantized(c, p):
    """The reconstruction of every weight from the packed plan, [rows, cols] in 32 bits."""
    rows, cols, G, R_u = c["rows"], c["cols"], c["G"], p["R_u"]
    nc = cols // G
    a = p["action"].long()
    bits = torch.tensor([0, 8, 4, 3, 2, 0, 1], device=DEV)[a]
    per_row = torch.tensor([_bytes_per_group(i, G) for i in range(7)], device=DEV)[a]
    row = p["code_off"][:-1, None] + per_row[:, None] * torch.arange(R_u, device=DEV)               # [U, R_u] where a row's codes start
    i = torch.arange(G, device=DEV)
    last = p["codes"].numel() - 1
    bit = bits[:, None, None] * i                                                                    # [U, 1, G]
    first = row[:, :, None] + torch.where(a[:, None, None] == 5, i // 5, bit >> 3)
    low = p["codes"][first.clamp(max=last)].to(torch.int32)
    high = p["codes"][(first + 1).clamp(max=last)].to(torch.int32)
    q = ((low | (high << 8)) >> (bit & 7).to(torch.int32)) & ((1 << bits) - 1).to(torch.int32)[:, None, None]
    trit = (low // torch.tensor([1, 3, 9, 27, 81], dtype=torch.int32, device=DEV)[i % 5]) % 3
    kind = a[:, None, None]
    q = torch.where(kind == 5, trit - 1, torch.where(kind == 6, 2 * q - 1, q)).float()
    w = p["offset"].reshape(-1, R_u, 1) + q * p["scale"].reshape(-1, R_u, 1)
    W = p["W"].float().reshape(rows // R_u, R_u, nc, G).permute(0, 2, 1, 3).reshape(-1, R_u, G)
    w = torch.where(kind == 0, W, w)
    return w.reshape(rows // R_u, nc, R_u, G).permute(0, 2, 1, 3).reshape(rows, cols)


def _act(word, x):
    """The activation and its slope."""
    if word == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return x * s, s * (1.0 + x * (1.0 - s))
    if word == "gelu":
        phi = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
        return x * phi, phi + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (x + 0.044715 * x * x * x))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * x * x)


def _plain(s):
    c = s["case"]
    op, dtype = c["op"], _type(c["dtype"])
    if op == "tokens8":
        return list(_eight(s["X"].float(), c["G"]))
    if op == "gated_grad":
        dh, g, u = s["dH"].float(), s["G"].float(), s["U"].float()
        y, slope = _act(c["act"], g)
        dg, du = dh * u * slope, dh * y
        dx = torch.matmul(dg, _dequantized(c, s["plans"][0])) + torch.matmul(du, _dequantized(c, s["plans"][1]))
        return [dx.to(dtype), dg.to(dtype), du.to(dtype)]
    x = s["X"].float() if op == "gated" else s["q"].float()
    each = [torch.matmul(x, _dequantized(c, p).t()) for p in s["plans"]]
    if op != "gated":
        each = [y * s["sigma"][:, None] for y in each]
    if op == "project8":
        return [each[0].to(dtype)]
    h = (_act(c["act"], each[0])[0] * each[1]).to(dtype)
    return [h] + ([y.to(dtype) for y in each] if c["save"] else [])


def _kept(s):
    """What a program keeps between its calls: the plans' descriptors and their forms for serving, workspaces, outputs."""
    import paper_2605_26660_amd as wq

    if "kept" not in s:
        c = s["case"]
        op, T, rows, dtype = c["op"], c["tokens"], c["rows"], _type(c["dtype"])
        plans = [wq.Packed(p["W"], c["G"], c["unit_rows"], p["action"], p["code_off"], p["codes"], p["scale"], p["offset"]) for p in s.get("plans", [])]
        k = dict(out=torch.empty(T, rows, dtype=dtype, device=DEV))
        if op == "tokens8":
            k["out"] = wq.Tokens8.empty(T, c["cols"], c["G"], DEV)
        elif op in ("project8", "gated8"):
            k["plans"] = [wq.Serving(p) for p in plans]
            k["tokens"] = wq.Tokens8(s["q"], s["sigma"], s["sums"], c["cols"], c["G"])
        else:
            k["plans"] = plans
            k["ws"] = wq.gated_workspace(*plans, s["X"] if op == "gated" else s["dH"], grad=op == "gated_grad")
            if op == "gated_grad":
                k["out"] = (torch.empty(T, c["cols"], dtype=dtype, device=DEV), torch.empty_like(s["G"]), torch.empty_like(s["U"]))
            elif c["save"]:
                k["save"] = (torch.empty_like(k["out"]), torch.empty_like(k["out"]))
        s["kept"] = k
    return wq, s["kept"]


def run(s):
    if not own:
        return _plain(s)
    c = s["case"]
    wq, k = _kept(s)
    if c["op"] == "tokens8":
        t = wq.windq_tokens8(s["X"], c["G"], out=k["out"])
        return [t.codes, t.scale, t.sums]
    if c["op"] == "project8":
        return [wq.windq_project8(k["plans"][0], k["tokens"], out=k["out"])]
    if c["op"] == "gated8":
        return [wq.windq_gated8(*k["plans"], k["tokens"], act=c["act"], out=k["out"])]
    if c["op"] == "gated":
        return [wq.windq_gated(*k["plans"], s["X"], act=c["act"], save=k.get("save"), ws=k["ws"], out=k["out"]), *k.get("save", ())]
    return list(wq.windq_gated_grad(*k["plans"], s["dH"], s["G"], s["U"], act=c["act"], ws=k["ws"], outs=k["out"]))


def work(case):
    rows, cols, T, G, op = (case[k] for k in ("rows", "cols", "tokens", "G", "op"))
    eb = 4 if case["dtype"] == "f32" else 2
    eight = T * (cols + 4)
    if op == "tokens8":
        return {"bytes": T * cols * eb + eight + 4 * T * (cols // _block(G)), "flops": 4.0 * T * cols}
    mix = POLICY if case["plan"] == "policy" else (1 / 7,) * 7
    weights = rows * cols * sum(share * (eb if a == 0 else (_bytes_per_group(a, G) + 8) / G) for a, share in enumerate(mix))
    if op == "project8":
        return {"bytes": weights + eight + T * rows * eb, "flops": 2.0 * T * rows * cols}
    flops = 4.0 * T * rows * cols + 10.0 * T * rows
    if op == "gated8":
        return {"bytes": 2 * weights + eight + T * rows * eb, "flops": flops}
    if op == "gated":
        return {"bytes": 2 * weights + T * (cols + rows * (3 if case["save"] else 1)) * eb, "flops": flops}
    return {"bytes": 2 * weights + T * (cols + 5 * rows) * eb, "flops": flops}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_weights(c, p):
    rows, cols, G, R_u = c["rows"], c["cols"], c["G"], p["R_u"]
    W = p["W"].double().clone()
    action, off = p["action"].cpu().numpy(), p["code_off"].cpu().numpy()
    scale, offset = p["scale"].double().reshape(-1, R_u, 1), p["offset"].double().reshape(-1, R_u, 1)
    for u, a in enumerate(action.tolist()):
        if a == 0:
            continue
        nb = _bytes_per_group(a, G)
        data = p["codes"][off[u]:off[u] + nb * R_u].reshape(R_u, nb).long()
        if a == 5:
            q = torch.stack([data // 3 ** k % 3 for k in range(5)], 2).reshape(R_u, -1)[:, :G] - 1
        else:
            b = {1: 8, 2: 4, 3: 3, 4: 2, 6: 1}[a]
            q = torch.stack([(data >> k) & 1 for k in range(8)], 2).reshape(R_u, G, b)
            q = sum(q[:, :, k] << k for k in range(b))
            q = 2 * q - 1 if a == 6 else q
        r0, c0 = u // (cols // G) * R_u, u % (cols // G) * G
        W[r0:r0 + R_u, c0:c0 + G] = q.double() * scale[u] + (0.0 if a in (5, 6) else offset[u])
    return W


def _exact_act(word, x):
    if word == "silu":
        return x * torch.sigmoid(x)
    return torch.nn.functional.gelu(x, approximate="tanh" if word == "gelu_tanh" else "none")


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "tokens8":
        return [None, s["X"].double().abs().amax(1) / 127.0, None]
    if op == "gated_grad":
        g, u = s["G"].double().requires_grad_(), s["U"].double().requires_grad_()
        dg, du = torch.autograd.grad(_exact_act(case["act"], g) * u, [g, u], s["dH"].double())
        return [dg @ _exact_weights(case, s["plans"][0]) + du @ _exact_weights(case, s["plans"][1]), dg, du]
    x = s["X"].double() if op == "gated" else s["q"].double() * s["sigma"].double()[:, None]
    each = [x @ _exact_weights(case, p).t().contiguous() for p in s["plans"]]
    if op == "project8":
        return each
    return [_exact_act(case["act"], each[0]) * each[1]] + (each if case["save"] else [])
