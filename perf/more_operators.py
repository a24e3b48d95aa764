"""Timed cases of what stands around a layer of experts in a training step and an answer: the layer norm before it and its
gradient, the router's balance loss and its gradient, the norm of all gradients and their clipping, and products of matrices in
microscaled 4-bit floating point.

Every operator is here twice: in its plain form (elementary torch operations in 32 bits) and, where `own` is true, as the calls a
user makes of the library.  Activations are N(0, 1) with an offset and a few channels that are far larger than the others, as the
rows before a norm have them; weights N(0, 1/K); a router's logits N(0, 1) around a bias per expert.
"""
import math

import torch

own = False


# ---- cases -----------------------------------------------------------------------------------------------------

def _norm(T, D, grad, x="bf16", y="bf16"):
    return {"op": "norm", "T": T, "D": D, "grad": grad, "x": x, "y": y}


def _balance(T, E, k, padding, grad):
    return {"op": "balance", "T": T, "E": E, "k": k, "padding": padding, "grad": grad}


def _clip(tensors, matrix, vector, bf16, ratio):
    """`tensors` gradients: every third a matrix of `matrix` values or so, the others vectors of `vector` or so."""
    return {"op": "clip", "tensors": tensors, "matrix": matrix, "vector": vector, "bf16": bf16, "ratio": ratio}


def _round(R, K, x="bf16", y="bf16"):
    return {"op": "round", "R": R, "K": K, "x": x, "y": y}


def _product(T, E, k, N, K, act="none", out="bf16"):
    return {"op": "product", "T": T, "E": E, "k": k, "N": N, "K": K, "act": act, "out": out}


def listed():
    def named(name, c):
        return {"name": name, **c}
    return [
        # the norm while one token is answered: the latency of the smallest call
        named("norm_token", _norm(1, 2048, False)),
        # the norm of a training step's forward pass
        named("norm_batch", _norm(16384, 2048, False)),
        # its gradient, with those of gamma and beta
        named("norm_batch_grad", _norm(16384, 2048, True)),
        # the gradient on 32-bit rows of an odd length
        named("norm_odd_grad", _norm(4099, 1001, True, x="f32", y="f32")),
        # the balance loss of a training step, some rows padding whose logits are all masked
        named("balance_batch", _balance(16384, 128, 8, 0.02, False)),
        # its gradient on the logits
        named("balance_batch_grad", _balance(16384, 64, 4, 0.0, True)),
        # the gradients of a layer of 8 experts of 2048 x 4096 weights in 32 bits
        named("clip_layer", _clip(24, 8 << 21, 2048, False, 0.1)),
        # the gradients of a model of many small tensors, some in 16 bits
        named("clip_many", _clip(300, 40000, 700, True, 0.5)),
        # weights of 16 matrices 4096 x 2048 to microscaled 4 bits and what the codes stand for
        named("mx4_round", _round(16 * 4096, 2048)),
        # training's shape or a prompt's: first product of the experts, tokens in bfloat16 read through the plan
        named("mx4_product_batch", _product(8192, 16, 4, 4096, 2048, act="relu")),
        # one token through one matrix
        named("mx4_product_token", _product(1, 1, 1, 4096, 4096)),
        # nothing a multiple of anything
        named("mx4_product_ragged", _product(1001, 7, 2, 777, 531, out="f32")),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length between lo and hi: mostly a multiple of 8, now and then any."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.3 else max(8, n // 8 * 8)


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "balance", "balance_grad", "clip", "round", "product", "product", "few"])
    types = ["bf16", "f32"]
    if kind.startswith("norm"):
        D = _size(rng, 64, 12288)
        return _norm(_log_int(rng, 1, min(16384, (1 << 25) // D)), D, kind == "norm_grad", rng.choice(types), rng.choice(types))
    if kind.startswith("balance"):
        k = rng.choice([1, 2, 4, 6, 8])
        return _balance(_log_int(rng, 1, 16384), max(k, _log_int(rng, 4, 256)), k, rng.choice([0.0, 0.05]), kind == "balance_grad")
    if kind == "clip":
        n = _log_int(rng, 1, 400)
        return _clip(n, _log_int(rng, 64, (1 << 26) // n), _log_int(rng, 1, 16384), rng.random() < 0.5, rng.choice([0.01, 0.5, 2.0]))
    k = rng.choice([1, 2, 4, 6, 8])
    E = max(k, _log_int(rng, 1, 64))
    N, K = _size(rng, 256, 4096), _size(rng, 256, 4096)
    if kind == "round":
        return _round(_log_int(rng, 1, (1 << 26) // K), K, rng.choice(types), rng.choice(types))
    E = min(E, 32, (1 << 27) // (N * K))                        # the weights fit beside their 32-bit copies
    k = min(k, E)
    if kind == "few":
        return _product(_log_int(rng, 1, 64), E, k, N, K, rng.choice(["none", "relu"]))
    rows = min(32768, (1 << 38) // (N * K))                     # no more work than the largest listed case
    return _product(max(1, _log_int(rng, 256, rows) // k), E, k, N, K, rng.choice(["none", "relu", "relu6"]), rng.choice(types))


# ---- inputs ----------------------------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * scale


def _activations(g, T, D):
    """Rows with a mean of their own, and one channel in 64 of eight times the others' size."""
    channel = torch.where(torch.rand(D, generator=g, device="cuda") < 1 / 64, 8.0, 1.0)
    return (_normal(g, T, D) + 0.5 + _normal(g, T, 1, scale=0.25)) * channel


def _logits(g, T, E, padding=0.0):
    x = _normal(g, T, E) + _normal(g, E, scale=0.5)
    if padding:
        x = torch.where(torch.rand(T, 1, generator=g, device="cuda") < padding, -math.inf, x)
    return x.contiguous()


def _plan(g, T, E, k):
    """offsets and the token of each slot for random choices of k experts, and the longest group."""
    ids = _logits(g, T, E).topk(k, dim=1).indices.reshape(-1)
    order = torch.argsort(ids, stable=True)
    counts = torch.zeros(E, dtype=torch.int64, device="cuda").scatter_add_(0, ids, torch.ones_like(ids))
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    return offsets, (order // k).int(), max(1, int(counts.max()))


def _by_type(tensors, types=(torch.float32, torch.bfloat16)):
    return [v for v in ([t for t in tensors if t.dtype == kind] for kind in types) if v]


def _lengths(case):
    """How many values each gradient has: lengths that differ, a scalar among them."""
    n = []
    for i in range(case["tensors"]):
        size = case["matrix"] if i % 3 == 0 else case["vector"]
        n.append(max(1, size - (7 * i) % (size // 4 + 1)))
    return n


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "norm":
        T, D = case["T"], case["D"]
        s["x"] = _activations(g, T, D).to(_type(case["x"]))
        s["gamma"], s["beta"] = 1 + _normal(g, D, scale=0.2), _normal(g, D, scale=0.2)
        if case["grad"]:
            s["dy"] = _normal(g, T, D, scale=1 / math.sqrt(D)).to(_type(case["y"]))
            s["mean"], s["rstd"] = _moments(s["x"].float())
        return s
    if case["op"] == "balance":
        s["logits"] = _logits(g, case["T"], case["E"], case["padding"])
        top = s["logits"].topk(case["k"], dim=1)
        s["ids"] = torch.where(top.values == -math.inf, -1, top.indices).int()
        if case["grad"]:
            s["counts"] = _counts(s["ids"], case["E"])
            s["rows"] = (s["logits"].amax(1) > -math.inf).sum().int()
            s["dloss"] = torch.rand((), generator=g, device="cuda") * 0.01
        return s
    if case["op"] == "clip":
        s["grads"] = [_normal(g, n, scale=10.0 ** (i % 5 - 3)) for i, n in enumerate(_lengths(case))]
        if case["bf16"]:
            s["grads"] = [t.bfloat16() if i % 2 else t for i, t in enumerate(s["grads"])]
        # what is clipped lies one tensor behind the other, a buffer for each type
        s["flat"] = [torch.cat(v) for v in _by_type(s["grads"])]
        ends = {t.dtype: 0 for t in s["flat"]}
        s["out"] = []
        for t in s["grads"]:
            flat = next(f for f in s["flat"] if f.dtype == t.dtype)
            s["out"].append(flat[ends[t.dtype]:ends[t.dtype] + t.numel()])
            ends[t.dtype] += t.numel()
        s["max_norm"] = case["ratio"] * float(_total(s["grads"]))
        return s
    if case["op"] == "round":
        s["x"] = _activations(g, case["R"], case["K"]).to(_type(case["x"]))
        return s
    T, E, N, K = case["T"], case["E"], case["N"], case["K"]
    s["offsets"], s["tokens"], s["most"] = _plan(g, T, E, case["k"])
    s["x"] = _activations(g, T, K).bfloat16()
    parts = [_quantise(_normal(g, N, K, scale=K ** -0.5).bfloat16()) for _ in range(E)]
    s["wq"], s["wscales"] = (torch.stack([_pack(q) for q, _ in parts]), torch.stack([b for _, b in parts]))
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------

def _moments(x, eps=1e-5):
    mean = x.mean(1)
    c = x - mean.unsqueeze(1)
    return mean, 1 / torch.sqrt((c * c).mean(1) + eps)


def _plain_norm(s):
    x = s["x"].float()
    if not s["case"]["grad"]:
        mean, rstd = _moments(x)
        h = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
        return (h * s["gamma"] + s["beta"]).to(_type(s["case"]["y"])), mean, rstd
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(1)
    h = (x - s["mean"].unsqueeze(1)) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx.to(_type(s["case"]["x"])), (dy * h).sum(0), dy.sum(0)


def _counts(ids, E):
    flat = torch.where(ids < 0, E, ids).reshape(-1).long()
    return torch.zeros(E + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))[:E].int()


def _probabilities(x):
    m = x.amax(1, keepdim=True)
    open_ = m > -math.inf
    e = torch.exp(x - torch.where(open_, m, torch.zeros_like(m)))
    total = e.sum(1, keepdim=True)
    return e / torch.where(open_, total, torch.ones_like(total)), open_.sum()


def _plain_balance(s):
    E = s["case"]["E"]
    p, rows = _probabilities(s["logits"])
    counts = s["counts"] if s["case"]["grad"] else _counts(s["ids"], E)
    f = counts.float() / counts.sum().clamp(min=1).float()
    if s["case"]["grad"]:
        return s["dloss"] * E / s["rows"].clamp(min=1).float() * p * (f - (p * f).sum(1, keepdim=True))
    shares = p.sum(0) / rows.clamp(min=1).float()
    return E * (f * shares).sum(), counts, shares, rows.int()


def _total(grads):
    parts = torch.stack([torch.sum(t.float() * t.float(), dtype=torch.float64) for t in grads])
    return torch.sqrt(parts.sum())


def _plain_clip(s):
    total = _total(s["grads"])
    factor = torch.clamp(s["max_norm"] / total, max=1.0).float()
    return total.float(), [torch.cat(v) for v in _by_type([(t.float() * factor).to(t.dtype) for t in s["grads"]])]


def _quantise(x):
    """Codes [...][KB][32] (a bit of sign, three of magnitude) and scales [...][KB] of blocks of 32 values, rows filled up with zeros to whole
    128; a scale is the byte b of 2^(b - 127)."""
    v = torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % 128))
    v = v.reshape(*v.shape[:-1], -1, 32)
    top = v.abs().amax(-1)
    e = torch.frexp(top).exponent                                # top = m 2^e with 1/2 <= m < 1
    b = torch.where(top > 0, e - 3 + 127, torch.zeros_like(e)).clamp(min=0)
    r = torch.ldexp(v.abs(), (127 - b).unsqueeze(-1))
    code = torch.zeros_like(v, dtype=torch.uint8)
    for limit, ties_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (r >= limit) if ties_up else (r > limit)
    return code + 8 * torch.signbit(v), b.to(torch.uint8)


def _pack(code):
    """The library's layout: two codes a byte, the lower half first, [...][16 KB]."""
    q = code.reshape(*code.shape[:-2], -1, 2)
    return (q[..., 0] | (q[..., 1] << 4)).to(torch.uint8)


_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values(code, b):
    """What codes and scales stand for, [...][32 KB] in 32 bits."""
    table = torch.tensor(_MAGNITUDES + tuple(-m for m in _MAGNITUDES), device=code.device)
    return torch.ldexp(table[code.int()], (b.int() - 127).unsqueeze(-1)).flatten(-2)


def _plain_round(s):
    return _values(*_quantise(s["x"]))[:, :s["case"]["K"]].to(_type(s["case"]["y"]))


def _act(v, act):
    return v if act == "none" else v.clamp(min=0) if act == "relu" else v.clamp(0, 6)


def _plain_product(s):
    c = s["case"]
    o = s["offsets"].long()
    slot = torch.arange(c["T"] * c["k"], device=o.device)
    e = (slot[:, None] >= o[None, 1:]).sum(1)
    at = o[:-1, None] + torch.arange(s["most"], device=o.device)
    there = (at < o[1:, None]).unsqueeze(2)
    x = _values(*_quantise(s["x"]))[s["tokens"].long()]
    x = torch.where(there, x[at.clamp(max=slot.numel() - 1)], torch.zeros((), device=x.device))
    w = torch.stack((s["wq"] & 15, s["wq"] >> 4), -1).reshape(*s["wscales"].shape, 32)
    y = torch.bmm(x, _values(w, s["wscales"]).transpose(1, 2).contiguous())[e, slot - o[e]]
    return _act(y, c["act"]).to(_type(c["out"]))


# ---- the library's calls -----------------------------------------------------------------------------------------

def _own(s):
    import paper_2006_02230_amd as P
    c = s["case"]
    if c["op"] == "norm":
        if c["grad"]:
            return tuple(P.layernorm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"]))
        return tuple(P.layernorm_fwd(s["x"], s["gamma"], s["beta"], out_dtype=_type(c["y"])))
    if c["op"] == "balance":
        if c["grad"]:
            return P.balance_bwd(s["logits"], s["counts"], s["rows"], s["dloss"])
        return tuple(P.balance(s["logits"], s["ids"]))
    if c["op"] == "clip":
        return P.clip_grads(s["grads"], s["max_norm"], out=s["out"]), s["flat"]
    x = P.mx4_quantise(s["x"])
    if c["op"] == "round":
        return P.mx4_dequantise(x, c["K"], out_dtype=_type(c["y"]))
    return P.mx4_gemm(x, P.Mx4(s["wq"], s["wscales"]), offsets=s["offsets"], rows=s["tokens"], act=c["act"], out_dtype=_type(c["out"]))


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "balance": _plain_balance, "clip": _plain_clip, "round": _plain_round,
            "product": _plain_product}[state["case"]["op"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def _bytes(name):
    return 4 if name == "f32" else 2


def work(case):
    if case["op"] == "norm":
        n, bx, by = case["T"] * case["D"], _bytes(case["x"]), _bytes(case["y"])
        if case["grad"]:
            return {"bytes": n * (2 * bx + by) + 8 * case["T"] + 12 * case["D"], "flops": 12 * n}
        return {"bytes": n * (bx + by) + 8 * case["T"] + 8 * case["D"], "flops": 8 * n}
    if case["op"] == "balance":
        n = case["T"] * case["E"]
        if case["grad"]:
            return {"bytes": 8 * n + 4 * case["E"] + 8, "flops": 8 * n}
        return {"bytes": 4 * n + 4 * case["T"] * case["k"] + 8 * case["E"] + 8, "flops": 5 * n}
    if case["op"] == "clip":
        n = _lengths(case)
        half = sum(n[1::2]) if case["bf16"] else 0
        return {"bytes": 2 * (4 * sum(n) - 2 * half) + 4, "flops": 3 * sum(n)}
    if case["op"] == "round":
        return {"bytes": case["R"] * case["K"] * (_bytes(case["x"]) + _bytes(case["y"])), "flops": 4 * case["R"] * case["K"]}
    T, E, N, K = case["T"], case["E"], case["N"], case["K"]
    M, steps = T * case["k"], -(-K // 128)
    used = E * (1 - (1 - 1 / E) ** M)                            # experts that M random choices reach, in the mean
    return {"bytes": 2 * T * K + used * N * steps * 68 + _bytes(case["out"]) * M * N + 4 * M, "flops": 2 * M * N * K}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _nearest(x):
    """The values that blocks of 32 along the rows of x are held as."""
    K = x.shape[-1]
    v = torch.nn.functional.pad(x.double(), (0, -K % 32)).unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2, min=-127))
    r = (v / unit).abs().clamp(max=6)
    step = torch.exp2(torch.floor(torch.log2(r.clamp(min=1))) - 1)          # one bit behind the first, halves below 1
    return (torch.sign(v) * torch.round(r / step) * step * unit).flatten(-2)[..., :K]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, gamma = s["x"].double(), s["gamma"].double()
        if not case["grad"]:
            var, mean = torch.var_mean(x, 1, correction=0)
            y = (x - mean[:, None]) / torch.sqrt(var + 1e-5)[:, None] * gamma + s["beta"].double()
            return y, mean, torch.rsqrt(var + 1e-5)
        h = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        dy = s["dy"].double()
        g = dy * gamma
        along = torch.linalg.vecdot(g, h)[:, None] / case["D"]
        return s["rstd"].double()[:, None] * (g - g.mean(1, keepdim=True) - along * h), torch.linalg.vecdot(dy, h, dim=0), dy.sum(0)
    if case["op"] == "balance":
        x = s["logits"].double()
        p = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)       # a row without an open expert has no probabilities
        if case["grad"]:
            f = s["counts"].double() / max(1, int(s["counts"].sum()))
            return float(s["dloss"]) * case["E"] / max(1, int(s["rows"])) * (p * f - p * (p @ f)[:, None])
        counts = torch.stack([(s["ids"] == e).sum() for e in range(case["E"])]).double()
        shares = p.sum(0) / max(1, int((x > -math.inf).any(1).sum()))
        return case["E"] * torch.dot(counts / counts.sum().clamp(min=1), shares), None, shares, None
    if case["op"] == "clip":
        total = math.sqrt(sum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["grads"]))
        return total, [torch.cat([t.double() * min(1.0, s["max_norm"] / total) for t in v]) for v in _by_type(s["grads"])]
    if case["op"] == "round":
        return _nearest(s["x"])
    rows, o, parts = s["tokens"].long(), s["offsets"].tolist(), []
    x = _nearest(s["x"])
    magnitude = torch.tensor(_MAGNITUDES, dtype=torch.float64, device="cuda")
    i = torch.arange(case["K"], device="cuda")
    for e in range(case["E"]):
        code = s["wq"][e][:, i // 2].int() >> 4 * (i % 2)
        w = magnitude[(code & 7).long()] * torch.exp2(s["wscales"][e][:, i // 32].double() - 127)
        v = x[rows[o[e]:o[e + 1]]] @ torch.where((code & 8) > 0, -w, w).T
        if case["act"] != "none":
            v = torch.relu(v) if case["act"] == "relu" else torch.relu(v) - torch.relu(v - 6)
        parts.append(v)
    return torch.cat(parts)
