"""The 8-bit operators of pruned language-model layers: what a program that serves them calls, and their plain forms.

``norm``    root-mean-square norm with the residual's addition, output in 8-bit integers with a scale for each token
``gated``   SiLU(gate) * up in 8-bit integers with a scale for each token (in front of a gated block's second product)
``rows``    activations as they are, in 8-bit integers with a scale for each token
``linear``  product of such activations with column-wise N:M pruned 8-bit weights with a scale for each channel
"""
import math

import torch

own = False   # True: the framework's operators, False: their plain forms

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5
_LARGEST = 2.0 * 8192 * 4096 * 12288   # operations of the largest listed product, pruned columns counted
_CELLS = 8192 * 8192                    # elements of the largest listed norm


def _norm(name, tokens, h, dtype, residual=True):
    return {"name": name, "kind": "norm", "tokens": tokens, "h": h, "dtype": dtype, "residual": residual}


def _rows(name, kind, tokens, h, dtype):
    return {"name": name, "kind": kind, "tokens": tokens, "h": h, "dtype": dtype}


def _linear(name, tokens, k, c_out, n, m, tile, dtype, bias=False):
    return {"name": name, "kind": "linear", "tokens": tokens, "k": k, "c_out": c_out, "n": n, "m": m, "tile": tile, "dtype": dtype,
            "bias": bias}


def listed():
    return [
        # one token of one sequence: the smallest call, latency counts
        _norm("norm_1x4096_bf16", 1, 4096, "bf16"),
        # a ragged batch of a small model in 32 bits, rows that are no multiple of 16 bytes, first layer (no residual yet)
        _norm("norm_333x1001_f32", 333, 1001, "f32", residual=False),
        # a long prompt of a large model
        _norm("norm_8192x8192_bf16", 8192, 8192, "bf16"),
        # one token inside a gated block
        _rows("gated_1x12288_bf16", "gated", 1, 12288, "bf16"),
        # a prompt inside a gated block
        _rows("gated_4096x12288_bf16", "gated", 4096, 12288, "bf16"),
        # attention output of a few dozen tokens of odd width, and of a prompt
        _rows("rows_77x1003_f16", "rows", 77, 1003, "f16"),
        _rows("rows_4096x4096_bf16", "rows", 4096, 4096, "bf16"),
        # one token through a projection at 2:4: the retained weights are all that has to be read
        _linear("linear_1_4096x4096_2of4_bf16", 1, 4096, 4096, 2, 4, 64, "bf16"),
        # a few sequences in step, 75 % of the columns pruned, 32-bit output with a bias
        _linear("linear_6_8192x2048_1of4_f32", 6, 8192, 2048, 1, 4, 32, "f32", bias=True),
        # a batch of sequences; nothing a multiple of a tile
        _linear("linear_45_1000x1001_2of8_f16", 45, 1000, 1001, 2, 8, 8, "f16", bias=True),
        # an unpruned layer, a short prompt
        _linear("linear_512_2048x2048_dense_bf16", 512, 2048, 2048, 4, 4, 64, "bf16"),
        # a long prompt through the widest projection
        _linear("linear_8192_4096x12288_2of4_bf16", 8192, 4096, 12288, 2, 4, 64, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "gated", "rows", "linear", "linear", "linear"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind != "linear":
        h = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            h = max(64, h // 64 * 64)
        tokens = _log(rng, 1, max(1, min(8192, _CELLS // (4 * h))))
        case = {"kind": kind, "tokens": tokens, "h": h, "dtype": dtype}
        return case | {"residual": rng.random() < 0.7} if kind == "norm" else case
    n, m = rng.choice(((2, 4), (2, 4), (1, 4), (3, 4), (2, 8), (4, 8), (1, 1)))
    tile = rng.choice((8, 16, 32, 64, 64, 128))
    k, c_out = _log(rng, 256, 12288), _log(rng, 256, 12288)
    if rng.random() < 0.75:
        k, c_out = k // 64 * 64, c_out // 64 * 64
    most = max(1, min(8192, int(_LARGEST / (4.0 * k * c_out))))
    return {"kind": "linear", "tokens": _log(rng, 1, most), "k": k, "c_out": c_out, "n": n, "m": m, "tile": tile, "dtype": dtype,
            "bias": rng.random() < 0.5}


def _kept(k, n, m):
    return k // m * n + min(k % m, n)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dtype = _TYPES[case["dtype"]]
    tokens = case["tokens"]

    def normal(*shape):
        return torch.randn(shape, device=dev, generator=g)

    if case["kind"] != "linear":
        h = case["h"]
        # tokens of different magnitude, a few channels that stand out, one token of padding (zeros) in longer batches
        spread = torch.exp(0.5 * normal(tokens, 1)) * (1.0 + 8.0 * (torch.rand(h, device=dev, generator=g) < 0.01))
        if tokens > 16:
            spread[tokens // 2] = 0.0
        x = (normal(tokens, h) * spread).to(dtype)
        if case["kind"] == "norm":
            residual = (2.0 * normal(tokens, h) * spread).to(dtype) if case["residual"] else None
            return {"case": case, "x": x, "residual": residual, "weight": (1.0 + 0.2 * normal(h)).to(dtype)}
        if case["kind"] == "gated":
            return {"case": case, "gate": x, "up": (normal(tokens, h) * spread).to(dtype)}
        return {"case": case, "x": x}

    k, c_out, n, m, tile = case["k"], case["c_out"], case["n"], case["m"], case["tile"]
    n_tiles, kk = -(-c_out // tile), _kept(k, n, m)
    # the retained columns of each tile and group: `n` of `m` at random, ascending (a short last group keeps at most `n`)
    order = torch.rand((n_tiles, -(-k // m) * m), device=dev, generator=g)
    order[:, k:] = 2.0
    rank = order.view(n_tiles, -1, m).argsort(-1).argsort(-1)
    keep = (rank < n).view(n_tiles, -1)[:, :k]
    indices = keep.nonzero()[:, 1].view(n_tiles, kk)
    values = torch.clamp(torch.round(40.0 * normal(c_out, kk)), -127, 127).to(torch.int8)
    by_row = indices.repeat_interleave(tile, 0)[:c_out]
    dense = torch.zeros((c_out, k), dtype=torch.int8, device=dev).scatter_(1, by_row, values)
    ld = -(-k // 16) * 16   # rows as the quantising operators lay them out
    xq = torch.clamp(torch.round(35.0 * normal(tokens, ld)), -127, 127).to(torch.int8)[:, :k]
    state = {"case": case, "xq": xq, "x_scale": 0.02 * torch.exp(0.5 * normal(tokens)), "dense": dense,
             "w_scale": 0.001 * torch.exp(0.3 * normal(c_out)), "bias": normal(c_out) if case["bias"] else None}
    if own:
        from paper_2507_17301_b200 import nm
        state["handle"] = nm.nm_q8_weights_import(values, state["w_scale"], indices.to(torch.uint16), k, n, m, tile)
    return state


def _values(q, scale, dtype):
    """What the 8-bit integers stand for, in the activations' type."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=dtype, device=q.device))


def _quantised(p, a):
    """Nearest integer to 127 p / a of each row, in 64 bits: 32 lose values next to a border."""
    return torch.round(127.0 * p / torch.where(a > 0, a, 1.0)[:, None])


def run(state):
    case = state["case"]
    kind, dtype = case["kind"], _TYPES[case["dtype"]]
    if own:
        from paper_2507_17301_b200 import nm
        if kind == "linear":
            return nm.nm_q8_linear(state["handle"], state["xq"], state["x_scale"], bias=state["bias"], out_dtype=dtype)
        if kind == "norm" and state["residual"] is not None:
            q, scale, residual = nm.nm_q8_rmsnorm(state["x"], state["weight"], _EPS, residual=state["residual"])
            return {"values": _values(q, scale, dtype), "scale": scale, "residual": residual}
        if kind == "norm":
            q, scale = nm.nm_q8_rmsnorm(state["x"], state["weight"], _EPS)
        elif kind == "gated":
            q, scale = nm.nm_q8_silu_mul(state["gate"], state["up"])
        else:
            q, scale = nm.nm_q8_rows(state["x"])
        return {"values": _values(q, scale, dtype), "scale": scale}

    if kind == "linear":
        acc = state["xq"].float() @ state["dense"].float().T
        y = acc * state["x_scale"][:, None] * state["w_scale"]
        return (y if state["bias"] is None else y + state["bias"]).to(dtype)
    out, factor = {}, 1.0
    if kind == "norm":
        s = state["x"].float()
        if state["residual"] is not None:
            out["residual"] = (s + state["residual"].float()).to(dtype)
            s = out["residual"].float()
        p = s.double() * state["weight"].double()
        factor = torch.rsqrt((s * s).mean(-1) + _EPS)
    elif kind == "gated":
        gate = state["gate"].double()
        p = gate / (1.0 + torch.exp(-gate)) * state["up"].double()
    else:
        p = state["x"].double()
    a = p.abs().amax(-1)
    out["scale"] = (a * factor / 127.0).float()
    out["values"] = _values(_quantised(p, a), out["scale"], dtype)
    return out


def work(case):
    b = torch.finfo(_TYPES[case["dtype"]]).bits // 8
    t = case["tokens"]
    if case["kind"] == "linear":
        k, c_out, kk = case["k"], case["c_out"], _kept(case["k"], case["n"], case["m"])
        read = t * k + 4 * t + c_out * kk + 4 * c_out + 4 * c_out * case["bias"]
        if case["n"] < case["m"]:
            read += 2 * -(-c_out // case["tile"]) * kk
        return {"bytes": read + t * c_out * b, "flops": 2 * t * c_out * kk}
    h = case["h"]
    if case["kind"] == "norm":
        return {"bytes": t * h * b * (3 if case["residual"] else 1) + h * b + t * h + 4 * t, "flops": 7 * t * h}
    return {"bytes": t * h * b * (2 if case["kind"] == "gated" else 1) + t * h + 4 * t, "flops": (12 if case["kind"] == "gated" else 4) * t * h}


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "linear":
        y = torch.einsum("tk,ok->to", state["xq"].double() * state["x_scale"].double()[:, None],
                         state["dense"].double() * state["w_scale"].double()[:, None])
        return y if state["bias"] is None else y + state["bias"].double()
    out = {}
    if case["kind"] == "norm":
        s = state["x"].double()
        if state["residual"] is not None:
            s = s + state["residual"].double()
            out["residual"] = s
            s = s.to(state["x"].dtype).double()   # the sum is held in the activations' type, and normed as it is held
        y = s / torch.sqrt(torch.sum(s * s, -1, keepdim=True) / case["h"] + _EPS) * state["weight"].double()
    elif case["kind"] == "gated":
        y = state["gate"].double() * torch.sigmoid(state["gate"].double()) * state["up"].double()
    else:
        y = state["x"].double()
    step = torch.linalg.vector_norm(y, ord=float("inf"), dim=-1, keepdim=True) / 127.0
    out["scale"] = step[:, 0]
    out["values"] = torch.where(step > 0, torch.round(y / torch.where(step > 0, step, 1.0)) * step, 0.0)
    return out
