"""Serving and training low-rank adapters beside a packed plan, as measurable cases.

Three operators.  `project`: a batch of tokens through one packed matrix, each token with the low-rank adapter of its own
request beside it.  `grad`: the way back of the same product, for the tokens and for the adapters.  `adamw`: one optimizer
step over many tensors, moments in 32 bits or in 8.  Shapes are those of the benchmark's decoder blocks and generic ones
of the same ranges.

A case holds: op; for the products rows, cols, G (chunk width), unit_rows (0 = whole columns), dtype, tokens, plan
("policy": the trained policy's mix at about 2 bits, "even": all seven treatments alike), adapters (how many), rank
(the longest), order ("runs": a request's tokens lie together, "mixed": any order) and none (every so many tokens one
without an adapter, 0 = never); for the step tensors (how many), numel (of the largest; the others are ragged fractions of it unless
"alike"), bits (of the moments), p and g (types of parameters and gradients), copy (a bfloat16 copy of the parameters is
written too), decay.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
F8 = torch.float8_e4m3fn
BLOCK = 256                                      # values that share a scale where moments are held in 8 bits
F8_MAX, F8_MIN = 448.0, 2.0 ** -9                # largest and smallest nonzero magnitude of that type
POLICY = (0.0866 / 4, 0.0866 / 4, 0.0866 / 4, 0.0866 / 4, 0.1565, 0.3654, 0.3915)
LEVELS = (0, 255, 15, 7, 3, 0, 0)                # largest code of the uniform treatments


def _product(name, op, rows, cols, tokens, G=128, unit_rows=0, dtype="bf16", plan="policy", adapters=0, rank=0, order="runs", none=0):
    c = dict(op=op, rows=rows, cols=cols, tokens=tokens, G=G, unit_rows=unit_rows, dtype=dtype, plan=plan, adapters=adapters,
             rank=rank, order=order, none=none)
    return dict(c, name=name) if name else c


def _step(name, tensors, numel, bits, p="f32", g="f32", alike=True, copy=False, decay=0.01):
    c = dict(op="adamw", tensors=tensors, numel=numel, bits=bits, p=p, g=g, alike=alike, copy=copy, decay=decay)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request through a 7B block's attention projection: latency
        _product("decode_1_attn_7b", "project", 4096, 4096, 1, adapters=4, rank=16),
        # a decoding step of 48 requests, each with an adapter of its own or none, through a 7B block's up projection
        _product("decode_48_up_7b", "project", 11008, 4096, 48, adapters=32, rank=32, order="mixed", none=7),
        # a prompt of 2000 tokens without adapters through a 7B block's down projection
        _product("prompt_2000_down_7b", "project", 4096, 11008, 2000),
        # the forward pass of a training step over 13B gate projections in tile units, four tasks in a batch
        _product("forward_4096_gate_13b", "project", 13824, 5120, 4096, unit_rows=128, adapters=4, rank=64),
        # a small fp32 layer of odd sizes, every treatment, requests in any order
        _product("layer_ragged_f32", "project", 1000, 1056, 77, G=96, dtype="f32", plan="even", adapters=5, rank=24, order="mixed", none=4),
        # the way back of a training step over a 7B block's up projection, one task
        _product("grad_2048_up_7b", "grad", 11008, 4096, 2048, adapters=1, rank=64),
        # the same for short sequences of sixteen tasks through an attention projection
        _product("grad_700_attn_7b", "grad", 4096, 4096, 700, adapters=16, rank=16, none=9),
        # the small layer's way back
        _product("grad_ragged_f32", "grad", 1000, 1056, 77, G=96, dtype="f32", plan="even", adapters=5, rank=24, order="mixed", none=4),
        # rank-16 adapters of every projection of a 7B stack, moments in 8 bits
        _step("adamw8_adapters_7b", 448, 65536, 8),
        # a whole 7B up projection, moments in 32 bits, bfloat16 gradients, the working copy written too
        _step("adamw32_up_7b", 1, 45088768, 32, g="bf16", copy=True),
        # the two adapters of one small layer: latency
        _step("adamw32_layer", 2, 8192, 32),
        # bfloat16 parameters of ragged sizes, moments in 8 bits
        _step("adamw8_ragged_bf16", 37, 700001, 8, p="bf16", g="bf16", alike=False, decay=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["project", "project", "grad", "grad", "adamw"])
    if op == "adamw":
        tensors = _log(rng, 1, 400)
        p = rng.choice(["f32", "f32", "bf16"])
        return _step(None, tensors, _log(rng, 1000, max(2000, min(30_000_000, 40_000_000 // tensors))), rng.choice([8, 32]), p=p,
                     g=rng.choice(["f32", "bf16"]), alike=rng.random() < 0.5, copy=p == "f32" and rng.random() < 0.5, decay=rng.choice([0.0, 0.01, 0.1]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    G = rng.choice([64, 64, 96, 128, 128, 128, 256])
    unit_rows = rng.choice([0, 0, 0, 128])
    tokens = _log(rng, 1, 4096)
    most = 13824 * 5120 if dtype == "bf16" else 1 << 22
    cols = G * _log(rng, 4, 11008 // G)
    rows = 8 * _log(rng, 32, max(33, min(13824, most // cols) // 8))
    if unit_rows:
        rows = max(unit_rows, rows // unit_rows * unit_rows)
    if dtype == "f32":
        tokens = min(tokens, 1024)
    if op == "grad":
        tokens = min(tokens, 2048)
    rank = 8 * _log(rng, 1, 8)
    return _product(None, op, rows, cols, tokens, G, unit_rows, dtype, rng.choice(["policy", "policy", "even"]),
                    min(_log(rng, 1, 32), tokens), rank, rng.choice(["runs", "mixed"]), rng.choice([0, 0, 5, 13]))


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


def _prepare_product(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    rows, cols, G, T = case["rows"], case["cols"], case["G"], case["tokens"]
    dtype = _type(case["dtype"])
    W = 0.02 * torch.randn(rows, cols, generator=g, device=DEV)
    W[:, torch.randperm(cols, generator=g, device=DEV)[:max(1, cols // 100)]] *= 5.0
    W = W.to(dtype)
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
    channel = torch.exp(0.5 * torch.randn(cols, generator=g, device=DEV))          # activations with channels of their own size
    s = dict(case=case, W=W, action=torch.from_numpy(action).to(DEV), code_off=torch.from_numpy(off).to(DEV), codes=codes,
             scale=scale.reshape(-1), offset=offset.reshape(-1), R_u=R_u,
             X=(torch.randn(T, cols, generator=g, device=DEV) * channel).to(dtype))
    if case["op"] == "grad":
        s["dY"] = (1e-3 * torch.randn(T, rows, generator=g, device=DEV)).to(dtype)
    n, r = case["adapters"], case["rank"]
    if n:
        # as they are after some training: A as drawn, B no longer zero; ranks differ from request to request
        s["a"] = (torch.randn(n, r, cols, generator=g, device=DEV) / math.sqrt(cols)).to(dtype)
        s["b"] = (0.02 * torch.randn(n, rows, r, generator=g, device=DEV)).to(dtype)
        ranks = np.array([max(1, r >> int(k)) for k in rng.randint(0, 3, n)])
        ranks[0] = r
        s["rank"] = torch.from_numpy(ranks.astype(np.int32)).to(DEV)
        s["alpha"] = torch.from_numpy((16.0 / ranks).astype(np.float32)).to(DEV)
        of = rng.randint(0, n, T) if case["order"] == "mixed" else np.sort(rng.randint(0, n, T))
        if case["none"]:
            of[::case["none"]] = -1
        s["adapter_of"] = torch.from_numpy(of.astype(np.int32)).to(DEV)
    return s


def _quantized(x):
    """x in blocks as (8-bit values, scales): every block over its largest magnitude; what is not zero does not become zero."""
    n = x.numel()
    blocks = torch.nn.functional.pad(x.reshape(-1), (0, -n % BLOCK)).reshape(-1, BLOCK)
    scale = blocks.abs().amax(1) * torch.tensor(1.0 / F8_MAX, dtype=torch.float32, device=DEV)
    whole = scale >= 2.0 ** -126
    inverse = torch.where(whole, 1.0 / scale, torch.zeros_like(scale))
    return (blocks * inverse[:, None]).to(F8), torch.where(whole, scale, torch.zeros_like(scale))


def _sizes(case):
    n, most = case["tensors"], case["numel"]
    return [most] * n if case["alike"] else [max(1, most * (1 + (i * 7) % 11) // (11 * (1 + i % 5)) - i) for i in range(n)]


def _prepare_step(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    sizes = _sizes(case)
    padded = [(n + BLOCK - 1) // BLOCK * BLOCK for n in sizes]      # a tensor of its own starts at an allocation's start
    total = sum(padded)
    s = dict(case=case, step=200, lr=1e-3, sizes=sizes)
    inside = torch.zeros(total, dtype=torch.bool, device=DEV)
    at = np.concatenate([[0], np.cumsum(padded)])
    edge = torch.zeros(total + 1, dtype=torch.int32, device=DEV)
    edge[torch.from_numpy(at[:-1]).to(DEV)] += 1
    edge.index_add_(0, torch.from_numpy(at[:-1] + np.array(sizes)).to(DEV), torch.full((len(sizes),), -1, dtype=torch.int32, device=DEV))
    inside = torch.cumsum(edge[:-1], 0) > 0
    p = 0.02 * torch.randn(total, generator=g, device=DEV) * inside
    size = torch.exp(torch.randn(total, generator=g, device=DEV))                 # gradients differ in size from weight to weight
    grad = 1e-3 * size * torch.randn(total, generator=g, device=DEV) * inside
    m = 2e-4 * size * torch.randn(total, generator=g, device=DEV) * inside
    r = 1e-3 * size * inside
    s["p"], s["g"] = p.to(_type(case["p"])), grad.to(_type(case["g"]))
    if case["bits"] == 8:
        m, s["m_scale"] = _quantized(m)
        r, s["v_scale"] = _quantized(r)
        s["m"], s["v"] = m.reshape(-1), r.reshape(-1)
    else:
        s["m"], s["v"] = m, r * r
    s["inside"] = inside
    if case["copy"]:
        s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
    s["clip"] = torch.full((1,), 0.75, device=DEV)                   # what clipping by the norm of all gradients left
    cut = lambda t, by=1: [t[a // by:a // by + (n + by - 1) // by] for a, n in zip(at[:-1].tolist(), sizes)]  # noqa: E731
    s["lists"] = {k: cut(s[k]) for k in ("p", "g", "m", "v", "copy") if k in s}
    s["lists"].update({k: cut(s[k], BLOCK) for k in ("m_scale", "v_scale") if k in s})
    return s


def prepare(case, seed):
    return _prepare_step(case, seed) if case["op"] == "adamw" else _prepare_product(case, seed)


# ------------------------------------------------------------------------------------------------ plain forms
def _dequantized(s):
    """The reconstruction of every weight from the packed plan, [rows, cols] in 32 bits."""
    c = s["case"]
    rows, cols, G, R_u = c["rows"], c["cols"], c["G"], s["R_u"]
    nc = cols // G
    a = s["action"].long()
    bits = torch.tensor([0, 8, 4, 3, 2, 0, 1], device=DEV)[a]
    per_row = torch.tensor([_bytes_per_group(i, G) for i in range(7)], device=DEV)[a]
    row = s["code_off"][:-1, None] + per_row[:, None] * torch.arange(R_u, device=DEV)               # [U, R_u] where a row's codes start
    i = torch.arange(G, device=DEV)
    last = s["codes"].numel() - 1
    bit = bits[:, None, None] * i                                                                    # [U, 1, G]
    first = row[:, :, None] + torch.where(a[:, None, None] == 5, i // 5, bit >> 3)
    low = s["codes"][first.clamp(max=last)].to(torch.int32)
    high = s["codes"][(first + 1).clamp(max=last)].to(torch.int32)
    q = ((low | (high << 8)) >> (bit & 7).to(torch.int32)) & ((1 << bits) - 1).to(torch.int32)[:, None, None]
    trit = (low // torch.tensor([1, 3, 9, 27, 81], dtype=torch.int32, device=DEV)[i % 5]) % 3
    kind = a[:, None, None]
    q = torch.where(kind == 5, trit - 1, torch.where(kind == 6, 2 * q - 1, q)).float()
    w = s["offset"].reshape(-1, R_u, 1) + q * s["scale"].reshape(-1, R_u, 1)
    W = s["W"].float().reshape(rows // R_u, R_u, nc, G).permute(0, 2, 1, 3).reshape(-1, R_u, G)
    w = torch.where(kind == 0, W, w)
    return w.reshape(rows // R_u, nc, R_u, G).permute(0, 2, 1, 3).reshape(rows, cols)


def _chosen(s):
    """[T, n, r]: the adapter of each token times its factor, and nothing for the others and past an adapter's rank; and where it is not zero."""
    n, r = s["case"]["adapters"], s["case"]["rank"]
    mine = s["adapter_of"][:, None, None] == torch.arange(n, device=DEV)[:, None]
    mine = mine & (torch.arange(r, device=DEV) < s["rank"][:, None])
    return mine * s["alpha"][:, None], mine


def _plain_project(s):
    x = s["X"].float()
    y = torch.matmul(x, _dequantized(s).t())
    if not s["case"]["adapters"]:
        return [y.to(s["X"].dtype)]
    n, r, T = s["case"]["adapters"], s["case"]["rank"], s["case"]["tokens"]
    factor, mine = _chosen(s)
    h = torch.matmul(x, s["a"].float().reshape(n * r, -1).t()).reshape(T, n, r)
    both = s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    y = y + torch.matmul((h * factor).reshape(T, n * r), both)
    return [y.to(s["X"].dtype), (h * mine).sum(1)]


def _plain_grad(s):
    x, dy = s["X"].float(), s["dY"].float()
    dx = torch.matmul(dy, _dequantized(s))
    n, r, T = s["case"]["adapters"], s["case"]["rank"], s["case"]["tokens"]
    factor, mine = _chosen(s)
    a = s["a"].float().reshape(n * r, -1)
    b = s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    h = torch.matmul(x, a.t()).reshape(T, n, r) * factor
    dh = (torch.matmul(dy, b.t()).reshape(T, n, r) * factor).reshape(T, n * r)
    dx = dx + torch.matmul(dh, a)
    da = torch.matmul(dh.t(), x).reshape(n, r, -1)
    db = torch.matmul(h.reshape(T, n * r).t(), dy).reshape(n, r, -1).permute(0, 2, 1).contiguous()
    return [dx.to(s["dY"].dtype), da, db]


def _rates(s):
    """The step's constants, in 32 bits as they enter: decay, size of the step, 1 / sqrt of the second moment's correction."""
    b1, b2, t = 0.9, 0.999, s["step"]
    return 1.0 - s["lr"] * s["case"]["decay"], s["lr"] / (1.0 - b1 ** t), 1.0 / math.sqrt(1.0 - b2 ** t)


def _plain_step(s):
    b1, b2, eps = 0.9, 0.999, 1e-8
    decay, size, inverse = _rates(s)
    eight = s["case"]["bits"] == 8
    g = s["g"].float() * s["clip"]
    m, v = s["m"].float(), s["v"].float()
    if eight:
        m = (m.reshape(-1, BLOCK) * s["m_scale"][:, None]).reshape(-1)
        v = (v.reshape(-1, BLOCK) * s["v_scale"][:, None]).reshape(-1)
        v = v * v                                                    # what is held in 8 bits is its root
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * g) * (1.0 - b2)
    root = torch.sqrt(v)
    p = s["p"].float() * decay - (m / (root * inverse + eps)) * size
    s["p"].copy_(p)
    if "copy" in s:
        s["copy"].copy_(p)
    if eight:
        m8, s["m_scale"][:] = _quantized(m)
        r8, s["v_scale"][:] = _quantized(root)
        small = (r8.float() == 0) & (root.reshape(-1, BLOCK) > 0) & (s["v_scale"] > 0)[:, None]
        r8 = torch.where(small, torch.full_like(root.reshape(-1, BLOCK), F8_MIN), r8.float()).to(F8)
        s["m"].copy_(m8.reshape(-1))
        s["v"].copy_(r8.reshape(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _kept(s):
    """What a program keeps between its calls: the plan's and the adapters' descriptors (addresses and sizes, nothing computed), workspaces, outputs."""
    import paper_2605_26660_amd as wq

    if "kept" not in s:
        c = s["case"]
        if c["op"] == "adamw":
            t = s["lists"]
            s["kept"] = wq.AdamwItems(t["p"], t["g"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale"), t.get("copy"))
        else:
            T, n, r = c["tokens"], c["adapters"], c["rank"]
            packed = wq.Packed(s["W"], c["G"], c["unit_rows"], s["action"], s["code_off"], s["codes"], s["scale"], s["offset"])
            adapters = wq.Adapters(s["a"], s["b"], s["alpha"], s["rank"]) if n else None
            ws = wq.project_workspace(packed, s["X"], adapters, grad=c["op"] == "grad")
            if c["op"] == "project":
                outs = (torch.empty(T, c["rows"], dtype=s["X"].dtype, device=DEV), torch.empty(T, r, device=DEV) if n else None)
            else:
                outs = (torch.empty_like(s["X"]), torch.empty(n, r, c["cols"], device=DEV), torch.empty(n, c["rows"], r, device=DEV))
            s["kept"] = packed, adapters, ws, outs
    return wq, s["kept"]


def run(s):
    c = s["case"]
    if c["op"] == "adamw":
        if own:
            wq, items = _kept(s)
            wq.windq_adamw(items, s["step"], s["lr"], 0.9, 0.999, 1e-8, c["decay"], grad_scale=s["clip"])
        else:
            _plain_step(s)
        return [s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if k in s]
    if not own:
        return _plain_project(s) if c["op"] == "project" else _plain_grad(s)
    wq, (packed, adapters, ws, outs) = _kept(s)
    if c["op"] == "grad":
        return list(wq.windq_project_grad(packed, s["dY"], s["X"], adapters, s["adapter_of"], ws=ws, outs=outs))
    y, h = outs
    if adapters is None:
        return [wq.windq_project(packed, s["X"], ws=ws, out=y)]
    return [wq.windq_project(packed, s["X"], adapters, s["adapter_of"], h=h, ws=ws, out=y), h]


def work(case):
    if case["op"] == "adamw":
        total = sum(_sizes(case))
        each = 2 * (4 if case["p"] == "f32" else 2) + (4 if case["g"] == "f32" else 2) + 2 * case["copy"]
        each += 4 * (1 + 4 / BLOCK) if case["bits"] == 8 else 16
        return {"bytes": total * each, "flops": total * 14}
    rows, cols, T, G, n, r = (case[k] for k in ("rows", "cols", "tokens", "G", "adapters", "rank"))
    eb = 4 if case["dtype"] == "f32" else 2
    mix = POLICY if case["plan"] == "policy" else (1 / 7,) * 7
    weights = rows * cols * sum(share * (eb if a == 0 else (_bytes_per_group(a, G) + 8) / G) for a, share in enumerate(mix))
    used = min(n, T)
    mean = r * 7 / 12                                # ranks are the longest, half and a quarter of it alike
    side = used * mean * (rows + cols) * eb
    if case["op"] == "project":
        return {"bytes": weights + side + T * (cols + rows) * eb + (T * r * 4 if n else 0),
                "flops": 2.0 * T * rows * cols + (2.0 * T * mean * (rows + cols) if n else 0)}
    return {"bytes": weights + side + T * (2 * cols + rows) * eb + n * r * (rows + cols) * 4,
            "flops": 2.0 * T * rows * cols + 2.0 * T * mean * 3 * (rows + cols)}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_weights(s):
    c = s["case"]
    rows, cols, G, R_u = c["rows"], c["cols"], c["G"], s["R_u"]
    W = s["W"].double().clone()
    action, off = s["action"].cpu().numpy(), s["code_off"].cpu().numpy()
    scale, offset = s["scale"].double().reshape(-1, R_u, 1), s["offset"].double().reshape(-1, R_u, 1)
    for u, a in enumerate(action.tolist()):
        if a == 0:
            continue
        nb = _bytes_per_group(a, G)
        data = s["codes"][off[u]:off[u] + nb * R_u].reshape(R_u, nb).long()
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


def _exact_product(s):
    c = s["case"]
    x, n, r, T = s["X"].double(), c["adapters"], c["rank"], c["tokens"]
    W = _exact_weights(s)
    if c["op"] == "project":
        y, h = x @ W.t().contiguous(), torch.zeros(T, max(1, r), dtype=torch.float64, device=DEV)
        for k in range(n):
            at, rk = torch.nonzero(s["adapter_of"] == k)[:, 0], int(s["rank"][k])
            h[at, :rk] = x[at] @ s["a"][k, :rk].double().t().contiguous()
            y[at] += float(s["alpha"][k]) * (h[at, :rk] @ s["b"][k, :, :rk].double().t().contiguous())
        return [y, h] if n else [y]
    dy = s["dY"].double()
    dx = dy @ W
    da = torch.zeros(n, r, c["cols"], dtype=torch.float64, device=DEV)
    db = torch.zeros(n, c["rows"], r, dtype=torch.float64, device=DEV)
    for k in range(n):
        at, rk, alpha = torch.nonzero(s["adapter_of"] == k)[:, 0], int(s["rank"][k]), float(s["alpha"][k])
        a, b = s["a"][k, :rk].double(), s["b"][k, :, :rk].double().contiguous()
        dh = alpha * (dy[at] @ b)
        dx[at] += dh @ a
        da[k, :rk] = dh.t().contiguous() @ x[at]
        db[k, :, :rk] = alpha * (dy[at].t().contiguous() @ (x[at] @ a.t().contiguous()))
    return [dx, da, db]


def _exact_eight(x, floor):
    """Nearest 8-bit values (ties to the even code) over each block's largest magnitude, found in the table of all of them."""
    table = torch.arange(127, dtype=torch.uint8, device=DEV).view(F8).double()
    x = x.reshape(-1, BLOCK)
    scale = x.abs().amax(1, keepdim=True) / F8_MAX
    t = x.abs() / torch.where(scale > 0, scale, torch.ones_like(scale))
    k = torch.searchsorted(table, t).clamp(1, 126)
    down, up = t - table[k - 1], table[k] - t
    k = torch.where((down < up) | ((down == up) & (k % 2 == 1)), k - 1, k)
    if floor:
        k = torch.where((k == 0) & (t > 0), torch.ones_like(k), k)
    return (table[k] * torch.sign(x)).reshape(-1), scale[:, 0]


def _exact_step(s):
    c = s["case"]
    eight = c["bits"] == 8
    g = s["g"].double() * s["clip"].double()
    m, v = s["m"].double(), s["v"].double()
    if eight:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = 0.9 * m + 0.1 * g
    v = 0.999 * v + 0.001 * g * g
    hat = m / (1 - 0.9 ** s["step"])
    p = s["p"].double() * (1 - s["lr"] * c["decay"]) - s["lr"] * hat / ((v / (1 - 0.999 ** s["step"])).sqrt() + 1e-8)
    if not eight:
        return [p, m, v] + ([p] if "copy" in s else [])
    (m8, ms), (r8, rs) = _exact_eight(m, False), _exact_eight(v.sqrt(), True)
    return [p, m8, r8, ms, rs] + ([p] if "copy" in s else [])


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_step(s) if case["op"] == "adamw" else _exact_product(s)
