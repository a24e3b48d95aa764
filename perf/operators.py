"""Timed cases of the layer of experts: the router and its plan, the products grouped by expert in the three
directions of training, the weighted sum over a token's experts, and the products with 4-bit weights that answer
single tokens.

Every operator is here twice: in its plain form (elementary torch operations in 32 bits) and, where `own` is true, as
the calls a user makes of the library.  Weights are N(0, 1/K), activations N(0, 1); a router's logits are N(0, 1)
around a bias per expert, so that the groups are as uneven as a trained router's.
"""
import math

import torch

own = False


# ---- cases -----------------------------------------------------------------------------------------------------

def _route(T, E, k, renorm, padding, grad):
    return {"op": "route", "T": T, "E": E, "k": k, "renorm": renorm, "padding": padding, "grad": grad}


def _combine(T, E, k, D, grad):
    return {"op": "combine", "T": T, "E": E, "k": k, "D": D, "grad": grad}


def _product(form, T, E, k, N, K, gather, act="none", out="bf16"):
    return {"op": "product", "form": form, "T": T, "E": E, "k": k, "N": N, "K": K, "gather": gather, "act": act, "out": out}


def _w4(T, E, k, N, K, group, zeros, act="none"):
    return {"op": "w4", "T": T, "E": E, "k": k, "N": N, "K": K, "group": group, "zeros": zeros, "act": act}


def listed():
    def named(name, c):
        return {"name": name, **c}
    return [
        # the router while one token is answered: the latency of the smallest call
        named("route_token", _route(1, 64, 4, True, 0.0, False)),
        # the router of a training step, some rows padding whose logits are all masked
        named("route_batch", _route(16384, 128, 8, True, 0.02, False)),
        # its gradient, weights taken from the softmax over all experts
        named("route_batch_grad", _route(16384, 64, 4, False, 0.0, True)),
        # the weighted sum at the end of a training step's forward pass
        named("combine_batch", _combine(8192, 64, 4, 2048, False)),
        # its gradient on rows of an odd length
        named("combine_odd_grad", _combine(4099, 16, 2, 1001, True)),
        # training, forward: first product of the experts, tokens read through the plan, ReLU on the way out
        named("product_fwd_batch", _product("fwd", 8192, 16, 4, 4096, 2048, True, act="relu")),
        # training, backward: the gradient of the rows through the second product, masked by the first one's ReLU
        named("product_dx_batch", _product("dx", 8192, 16, 2, 2048, 4096, False, act="relu")),
        # training, backward: the gradient of the weights in 32 bits, tokens read through the plan
        named("product_dw_batch", _product("dw", 8192, 8, 2, 4096, 2048, True, out="f32")),
        # a batch of single tokens: few rows an expert, every expert's weights read
        named("product_fwd_few", _product("fwd", 64, 64, 4, 1536, 2048, True)),
        # nothing a multiple of anything
        named("product_fwd_ragged", _product("fwd", 1001, 7, 1, 777, 531, True)),
        # one token through one matrix in 4 bits
        named("w4_token", _w4(1, 1, 1, 4096, 4096, 128, False)),
        # eight tokens through their experts' matrices in 4 bits
        named("w4_experts", _w4(8, 64, 4, 2048, 4096, 64, True, act="relu")),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length between lo and hi: mostly a multiple of 8, now and then any."""
    n = _log_int(rng, lo, hi)
    if rng.random() < 0.2:
        return n - (n == 3072)
    n = max(8, n // 8 * 8)
    return n - 8 * (n == 3072)


def draw(rng):
    kind = rng.choice(["route", "route_grad", "combine", "combine_grad", "fwd", "dx", "dw", "few", "w4", "w4_experts"])
    k = rng.choice([1, 2, 4, 6, 8])
    E = max(k, _log_int(rng, 4, 128))
    if kind.startswith("route"):
        return _route(_log_int(rng, 1, 16384), E, k, rng.random() < 0.5, rng.choice([0.0, 0.05]), kind == "route_grad")
    if kind.startswith("combine"):
        T = _log_int(rng, 1, 8192)
        return _combine(T, E, k, _size(rng, 64, min(4096, (1 << 26) // (T * k))), kind == "combine_grad")
    if kind == "w4":
        return _w4(_log_int(rng, 1, 24), 1, 1, _size(rng, 512, 8192), _size(rng, 512, 8192), rng.choice([32, 64, 128]), rng.random() < 0.5)
    N, K = _size(rng, 256, 4096), _size(rng, 256, 4096)
    if kind == "w4_experts":
        return _w4(_log_int(rng, 1, 16), min(E, 64), min(k, 4), N // 2 + 1 if N % 8 else N // 2, K, rng.choice([32, 64, 128]), rng.random() < 0.5,
                   rng.choice(["none", "relu"]))
    E = min(E, 32, (1 << 27) // (N * K))                        # the weights fit beside their 32-bit copies
    k = min(k, E)
    if kind == "few":
        return _product("fwd", _log_int(rng, 1, 128), E, k, N, K, rng.random() < 0.7)
    rows = min(32768, (1 << 38) // (N * K))                     # no more work than the largest listed case
    return _product(kind, max(1, _log_int(rng, 256, rows) // k), E, k, N, K, kind != "dx" and rng.random() < 0.5,
                    rng.choice(["none", "relu", "relu6"]) if kind != "dw" else "none", rng.choice(["bf16", "f32"]))


# ---- inputs ----------------------------------------------------------------------------------------------------

def _normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * scale


def _logits(g, T, E, padding=0.0):
    x = _normal(g, T, E) + _normal(g, E, scale=0.5)
    if padding:
        x = torch.where(torch.rand(T, 1, generator=g, device="cuda") < padding, -math.inf, x)
    return x.contiguous()


def _plan(g, T, E, k):
    """offsets, the token of each slot, the slot of each (token, j), for random choices of k experts."""
    ids = _logits(g, T, E).topk(k, dim=1).indices.reshape(-1)
    order = torch.argsort(ids, stable=True)
    counts = torch.zeros(E, dtype=torch.int64, device="cuda").scatter_add_(0, ids, torch.ones_like(ids))
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * k, device="cuda")
    return offsets, (order // k).int(), slots.reshape(T, k).int(), max(1, int(counts.max()))


def _quantise(w, group, asymmetric):
    """4-bit codes of w [E][N][K], scales and zero points a group of `group` inputs."""
    E, N, K = w.shape
    wg = torch.nn.functional.pad(w, (0, -K % group)).reshape(E, N, -1, group)
    lo, hi = wg.amin(-1).clamp(max=0), wg.amax(-1).clamp(min=0)
    if asymmetric:
        scale = ((hi - lo) / 15).bfloat16()
        zero = torch.where(scale > 0, -lo / scale.float().clamp(min=1e-30), torch.zeros_like(lo)).round().clamp(0, 15)
    else:
        scale = (torch.maximum(hi, -lo) / 7).bfloat16()
        zero = torch.full_like(lo, 8.0)
    q = (wg / scale.float().clamp(min=1e-30).unsqueeze(-1) + zero.unsqueeze(-1)).round().clamp(0, 15)
    return q.reshape(E, N, -1)[:, :, :K].to(torch.uint8), scale, zero.to(torch.uint8)


def _pack(q, scale, zero, group):
    """The library's layout of 4-bit weights: [E][N/16][K/128][lane][16 bytes], lane = 16 (block of 8 inputs) + row, the
    byte's word i and nibble p holding input 32 i + 8 (lane / 16) + 2 (p % 4) + p / 4; scales [E][N/16][K/group][16]."""
    E, N, K = q.shape
    pad = torch.nn.functional.pad
    q = pad(q, (0, -K % 128, 0, -N % 16), value=8)
    q = q.reshape(E, q.shape[1] // 16, 16, q.shape[2] // 128, 4, 4, 4, 2)   # E, tile, row, step, word, block, pair, half
    q = q.permute(0, 1, 3, 5, 2, 4, 7, 6).contiguous()                      # E, tile, step, block, row, word, half, pair
    q = q.reshape(*q.shape[:6], 4, 2)                                       # nibbles in order, two a byte
    q = (q[..., 0] | (q[..., 1] << 4)).reshape(E, q.shape[1], q.shape[2], 64, 16)
    groups = q.shape[2] * (128 // group)

    def tiles(v, fill):
        v = pad(v, (0, groups - v.shape[2], 0, -N % 16), value=fill)
        return v.reshape(E, -1, 16, groups).transpose(2, 3).contiguous()
    return q, tiles(scale, 0.0), tiles(zero, 8)


def _out_type(case):
    return torch.float32 if case.get("out") == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, E, k = case["T"], case["E"], case["k"]
    s = {"case": case}
    if case["op"] == "route":
        s["logits"] = _logits(g, T, E, case["padding"])
        if case["grad"]:
            s["dweights"] = _normal(g, T, k)
            s["ids"], s["weights"] = _choose(s["logits"], k, case["renorm"])
        return s
    s["offsets"], s["tokens"], s["slots"], s["most"] = _plan(g, T, E, k)
    M = T * k
    if case["op"] == "combine":
        s["y"] = _normal(g, M, case["D"]).bfloat16()
        s["weights"] = torch.softmax(_normal(g, T, k), 1)
        if case["grad"]:
            s["dout"] = _normal(g, T, case["D"]).bfloat16()
        return s
    N, K = case["N"], case["K"]
    if case["op"] == "w4":
        w = _normal(g, E, N, K, scale=K ** -0.5)
        q, scale, zero = _quantise(w, case["group"], case["zeros"])
        s["q"], s["scales"], zeros = _pack(q, scale, zero, case["group"])
        s["zeros"] = zeros if case["zeros"] else None
        s["x"] = _normal(g, T, K).bfloat16()
        return s
    if case["form"] != "dw":
        s["w"] = _normal(g, E, N, K, scale=(K if case["form"] == "fwd" else N) ** -0.5).bfloat16()
    if case["form"] != "dx":
        s["x"] = _normal(g, T if case["gather"] else M, K).bfloat16()
    if case["form"] != "fwd":
        s["dy"] = _normal(g, M, N).bfloat16()
    if case["form"] == "dx" and case["act"] != "none":
        h = _normal(g, M, K, scale=4.0).clamp(min=0)
        s["h"] = (h.clamp(max=6) if case["act"] == "relu6" else h).bfloat16()
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------

def _choose(logits, k, renorm):
    v, i = torch.sort(logits, dim=1, descending=True, stable=True)
    masked = v[:, :k] == -math.inf
    e = torch.exp(v - torch.where(v[:, :1] == -math.inf, torch.zeros_like(v[:, :1]), v[:, :1]))
    total = (e[:, :k] if renorm else e).sum(1, keepdim=True)
    w = torch.where(masked, torch.zeros_like(e[:, :k]), e[:, :k] / torch.where(total == 0, torch.ones_like(total), total))
    return torch.where(masked, -1, i[:, :k]).int(), w


def _plain_route(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    x = s["logits"]
    if c["grad"]:
        g, there = s["dweights"], s["ids"] >= 0
        g = torch.where(there, g, torch.zeros_like(g))
        at = s["ids"].clamp(min=0).long()
        spread = torch.zeros_like(x).scatter_add_(1, at, g)
        if c["renorm"]:
            p = torch.zeros_like(x).scatter_add_(1, at, torch.where(there, s["weights"], torch.zeros_like(g)))
        else:
            m = x.amax(1, keepdim=True)
            e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
            total = e.sum(1, keepdim=True)
            p = e / torch.where(total == 0, torch.ones_like(total), total)
        return p * (spread - (p * spread).sum(1, keepdim=True))
    ids, w = _choose(x, k, c["renorm"])
    flat = torch.where(ids < 0, E, ids).reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=x.device).scatter_add_(0, flat, torch.ones_like(flat))
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=x.device)
    offsets[1:] = counts[:E].cumsum(0)
    at = torch.arange(T * k, device=x.device)
    slots = torch.empty_like(at)
    slots[order] = at
    tokens = torch.where(at < offsets[E], order // k, -1)
    return ids, w, offsets.int(), tokens.int(), torch.where(ids < 0, -1, slots.reshape(T, k)).int()


def _plain_combine(s):
    rows = s["y"].float()[s["slots"].long()]
    if not s["case"]["grad"]:
        return (rows * s["weights"].unsqueeze(2)).sum(1).bfloat16()
    d = s["dout"].float().unsqueeze(1)
    dy = torch.empty_like(s["y"])
    dy[s["slots"].long()] = (d * s["weights"].unsqueeze(2)).bfloat16()
    return dy, (rows * d).sum(2)


def _act(v, act):
    return v if act == "none" else v.clamp(min=0) if act == "relu" else v.clamp(0, 6)


def _groups(s):
    """Row of each place of [E][most], whether it is one of the group's, and each slot's place."""
    o = s["offsets"].long()
    at = o[:-1, None] + torch.arange(s["most"], device=o.device)
    slot = torch.arange(s["case"]["T"] * s["case"]["k"], device=o.device)
    e = (slot[:, None] >= o[None, 1:]).sum(1)
    return at.clamp(max=slot.numel() - 1), at < o[1:, None], e, slot - o[e]


def _padded(rows, at, there):
    return torch.where(there.unsqueeze(2), rows.float()[at], torch.zeros((), device=rows.device))


def _plain_product(s):
    c = s["case"]
    at, there, e, place = _groups(s)
    if c["form"] == "fwd":
        x = s["x"].float()[s["tokens"].long()] if c["gather"] else s["x"]
        y = torch.bmm(_padded(x, at, there), s["w"].float().transpose(1, 2).contiguous())
        return _act(y[e, place], c["act"]).to(_out_type(c))
    if c["form"] == "dx":
        dx = torch.bmm(_padded(s["dy"], at, there), s["w"].float())[e, place]
        if c["act"] != "none":
            h = s["h"].float()
            open_ = (h > 0) if c["act"] == "relu" else (h > 0) & (h < 6)
            dx = torch.where(open_, dx, torch.zeros_like(dx))
        return dx.to(_out_type(c))
    x = s["x"].float()[s["tokens"].long()] if c["gather"] else s["x"]
    dw = torch.bmm(_padded(s["dy"], at, there).transpose(1, 2).contiguous(), _padded(x, at, there))
    return dw.to(_out_type(c))


def _unpack(s):
    """The weights [E][N][K] that the codes stand for."""
    c = s["case"]
    E, N, K, group = c["E"], c["N"], c["K"], c["group"]
    q = torch.stack((s["q"] & 15, s["q"] >> 4), -1)
    tiles, steps = q.shape[1], q.shape[2]
    q = q.reshape(E, tiles, steps, 4, 16, 4, 2, 4).permute(0, 1, 4, 2, 5, 3, 7, 6)   # E, tile, row, step, word, block, pair, half
    q = q.reshape(E, tiles * 16, steps * 128 // group, group).float()
    scale = s["scales"].float().transpose(2, 3).reshape(E, tiles * 16, -1, 1)
    zero = 8.0 if s["zeros"] is None else s["zeros"].float().transpose(2, 3).reshape(E, tiles * 16, -1, 1)
    return ((q - zero) * scale).reshape(E, tiles * 16, steps * 128)[:, :N, :K]


def _plain_w4(s):
    c = s["case"]
    at, there, e, place = _groups(s)
    x = _padded(s["x"].float()[s["tokens"].long()], at, there)
    y = torch.bmm(x, _unpack(s).transpose(1, 2).contiguous())[e, place]
    return _act(y, c["act"]).bfloat16()


# ---- the library's calls -----------------------------------------------------------------------------------------

def _own(s):
    import paper_2006_02230_amd as P
    c = s["case"]
    if c["op"] == "route":
        if c["grad"]:
            return P.route_bwd(s["logits"], s["ids"], s["weights"], s["dweights"], renorm=c["renorm"])
        return tuple(P.route(s["logits"], c["k"], renorm=c["renorm"]))
    if c["op"] == "combine":
        if c["grad"]:
            return P.combine_bwd_bf16(s["dout"], s["y"], s["slots"], s["weights"])
        return P.combine_bf16(s["y"], s["slots"], s["weights"])
    if c["op"] == "w4":
        return P.w4_gemm_bf16(s["x"], s["q"], s["scales"], c["N"], c["group"], zeros=s["zeros"], offsets=s["offsets"], rows=s["tokens"],
                              act=c["act"])
    rows = s["tokens"] if c["gather"] else None
    if c["form"] == "fwd":
        return P.grouped_gemm_bf16(s["x"], s["w"], s["offsets"], rows=rows, act=c["act"], out_dtype=_out_type(c))
    if c["form"] == "dx":
        return P.grouped_gemm_dx_bf16(s["dy"], s["w"], s["offsets"], h=s.get("h"), act=c["act"], out_dtype=_out_type(c))
    return P.grouped_gemm_dw_bf16(s["dy"], s["x"], s["offsets"], rows=rows, out_dtype=_out_type(c))


def run(state):
    if own:
        return _own(state)
    return {"route": _plain_route, "combine": _plain_combine, "product": _plain_product, "w4": _plain_w4}[state["case"]["op"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def _used(E, M):
    """Experts that M random choices reach, in the mean."""
    return E * (1 - (1 - 1 / E) ** M)


def work(case):
    T, E, k = case["T"], case["E"], case["k"]
    M = T * k
    if case["op"] == "route":
        if case["grad"]:
            return {"bytes": (4 if case["renorm"] else 8) * T * E + 12 * M, "flops": 6 * T * E}
        return {"bytes": 4 * T * E + 16 * M + 4 * (E + 1), "flops": 4 * T * E}
    if case["op"] == "combine":
        D = case["D"]
        if case["grad"]:
            return {"bytes": 4 * M * D + 2 * T * D + 12 * M, "flops": 3 * M * D}
        return {"bytes": 2 * M * D + 2 * T * D + 8 * M, "flops": 2 * M * D}
    N, K = case["N"], case["K"]
    flops = 2 * M * N * K
    if case["op"] == "w4":
        weights = _used(E, M) * N * (K / 2 + (3 if case["zeros"] else 2) * K / case["group"])
        return {"bytes": weights + 2 * T * K + 2 * M * N + 4 * M, "flops": flops}
    b = 4 if case["out"] == "f32" else 2
    x = 2 * K * (T if case["gather"] else M) + (4 * M if case["gather"] else 0)
    if case["form"] == "fwd":
        return {"bytes": x + 2 * _used(E, M) * N * K + b * M * N, "flops": flops}
    if case["form"] == "dx":
        return {"bytes": 2 * M * N + 2 * _used(E, M) * N * K + (b + (2 if case["act"] != "none" else 0)) * M * K, "flops": flops}
    return {"bytes": 2 * M * N + x + b * E * N * K, "flops": flops}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    k = case["k"]
    if case["op"] == "route":
        x = s["logits"].double()
        p = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)      # a row without an open expert has no probabilities
        if not case["grad"]:
            top = torch.topk(p, k, 1).values
            if case["renorm"]:
                top = torch.nan_to_num(top / top.sum(1, keepdim=True), nan=0.0)
            return None, top, None, None, None
        ids = s["ids"].long()
        chosen = torch.nn.functional.one_hot(ids.clamp(min=0), case["E"]).double() * (ids >= 0).unsqueeze(2)
        g = (chosen * s["dweights"].double().unsqueeze(2)).sum(1)
        if case["renorm"]:
            p = (chosen * s["weights"].double().unsqueeze(2)).sum(1)
        return p * g - p * (p * g).sum(1, keepdim=True)
    if case["op"] == "combine":
        w, slots = s["weights"].double(), s["slots"].long()
        if not case["grad"]:
            out = torch.zeros(case["T"], case["D"], dtype=torch.float64, device="cuda")
            for j in range(k):
                out += w[:, j:j + 1] * s["y"][slots[:, j]].double()
            return out
        dy = torch.empty(s["y"].shape, dtype=torch.float64, device="cuda")
        dw = torch.empty_like(w)
        for j in range(k):
            dy[slots[:, j]] = w[:, j:j + 1] * s["dout"].double()
            dw[:, j] = torch.linalg.vecdot(s["dout"].double(), s["y"][slots[:, j]].double())
        return dy, dw
    o = s["offsets"].tolist()
    gathered = case["op"] == "w4" or case["gather"]
    rows = s["tokens"].long()
    parts = []
    for e in range(case["E"]):
        a, b = o[e], o[e + 1]
        if case.get("form") != "dx":
            x = (s["x"][rows[a:b]] if gathered else s["x"][a:b]).double()
        if case["op"] == "w4":
            v = x @ _weights64(s, e).T
        elif case["form"] == "fwd":
            v = x @ s["w"][e].double().T
        elif case["form"] == "dx":
            v = s["dy"][a:b].double() @ s["w"][e].double()
            if case["act"] != "none":
                h = s["h"][a:b].double()
                v = v * (h > 0) * ((h < 6) if case["act"] == "relu6" else 1)
        else:
            v = s["dy"][a:b].double().T @ x
        if case.get("form") in (None, "fwd") and case["act"] != "none":
            v = torch.relu(v) if case["act"] == "relu" else torch.relu(v) - torch.relu(v - 6)
        parts.append(v)
    return torch.stack(parts) if case.get("form") == "dw" else torch.cat(parts)


def _weights64(s, e):
    """Expert e's weights in 64 bits, read from the layout place by place."""
    c = s["case"]
    n = torch.arange(c["N"], device="cuda")[:, None]
    k = torch.arange(c["K"], device="cuda")[None, :]
    j = k % 8
    word = (k % 128) // 32
    lane = 16 * ((k % 32) // 8) + n % 16
    nibble = j // 2 + 4 * (j % 2)
    byte = s["q"][e][n // 16, k // 128, lane, 4 * word + nibble // 2].int()
    q = torch.where(nibble % 2 == 1, byte >> 4, byte & 15).double()
    at = (n // 16, k // c["group"], n % 16)
    z = 8.0 if s["zeros"] is None else s["zeros"][e][at].double()
    return s["scales"][e][at].double() * (q - z)
