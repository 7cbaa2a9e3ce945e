"""The 8-bit layer around a model's norms, as cases that can be timed and compared: what runs where weights and activations have 8
bits each, with a scale for every token and every channel.

A case is a dict of plain values.  `kind` says which operator a pass goes through:

  "norm"     root-mean-square norm, with the residual's addition where there is one, in the tensors' own type; or with an output in 8
             bits with a scale for every row ("out": "codes")
  "quant"    rows to 8 bits with a scale each: activations that no norm precedes (an activation function and a second factor on the
             way), and weights
  "linear8"  y = residual + gate * act(x_scale w_scale (codes w^T) + bias), codes and weights in 8 bits

With `own` false, `run` computes them with elementary torch operations, with `own` true it calls the library.  Codes are returned as
the values they stand for.  Which code a value takes hangs on its distance from a border between two, so the plain form takes codes in 64 bits.

Sizes come from the workloads of `dvdq_inputs` (32760 tokens of a 480p clip, 118800 of a 720p one; channel widths 1536, 4608, 5120, 8960, 13824; heads of 128)
and from what surrounds such layers: conditioning vectors, text tokens, clips of few frames.
"""
import math

import torch

own = False

DEV = "cuda"
_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}

# The largest listed work of each kind: a drawn case stays below it.
_MAX_NORM = 118800 * 1536              # elements
_MAX_QUANT = 32760 * 8960
_MAX_FLOPS = 2 * 32760 * 13824 * 5120
_MAX_X = 32760 * 13824
_MAX_Y = 32760 * 8960


def _norm(name, rows, heads, C, residual, out, dtype="bf16", fused=False, rowsum=False):
    """heads: rows of C elements side by side in a token (0: one); fused: the rows are part of longer ones, q's heads in the output
    of the projection to q, k and v; rowsum: with the sum of every row's codes, for weights that have zero-points."""
    return {"name": name, "kind": "norm", "rows": rows, "heads": heads, "C": C, "residual": residual, "out": out, "dtype": dtype,
            "fused": fused, "rowsum": rowsum}


def _quant(name, rows, C, act, up, dtype="bf16"):
    """up: a second factor, which lies beside the first one in the rows of one product's output."""
    return {"name": name, "kind": "quant", "rows": rows, "C": C, "act": act, "up": up, "dtype": dtype}


def _linear8(name, M, K, N, act, bias, gate, residual, dtype="bf16"):
    """gate: rows of the gate (0 for none), each for M / gate tokens."""
    return {"name": name, "kind": "linear8", "M": M, "K": K, "N": N, "act": act, "bias": bias, "gate": gate, "residual": residual,
            "dtype": dtype}


def listed():
    return [
        # the smallest call: the token that a text decoder is at, added to the residual, normed and handed to an 8-bit product
        _norm("norm_one_token", 1, 0, 5120, True, "codes"),
        # q's heads, each normed by itself, where the fused projection left them
        _norm("norm_heads", 32760, 12, 128, False, "same", fused=True),
        # text tokens in 32 bits, a width that no vector divides, with the sums that weights with zero-points need
        _norm("norm_ragged", 2044, 0, 1533, True, "codes", "fp32", rowsum=True),
        # every token of the long clip, with the residual's addition
        _norm("norm_tokens", 118800, 0, 1536, True, "same"),
        # the middle of a gated feed-forward of a text encoder
        _quant("quant_gated_text", 512, 10240, "gelu_tanh", True, "fp16"),
        # the middle of a feed-forward layer at full length
        _quant("quant_tokens", 32760, 8960, "none", False),
        # a layer's weights, in 32 bits as a calibration keeps them
        _quant("quant_weights", 13824, 5120, "none", False, "fp32"),
        # the conditioning vector's modulation of both guidance branches: two rows, six outputs per channel
        _linear8("linear8_modulation", 2, 1536, 9216, "none", True, 0, False),
        # text tokens into the model's width
        _linear8("linear8_text_embed", 512, 4096, 5120, "gelu_tanh", True, 0, False),
        # a two-frame clip and one token of two guidance branches, gated into the residual, channel counts that no tile divides
        _linear8("linear8_ragged_gated", 6242, 1160, 1156, "none", True, 2, True, "fp16"),
        # the feed-forward layers at full length: up with its activation, down gated into the residual
        _linear8("linear8_ffn_up", 32760, 1536, 8960, "gelu_tanh", True, 0, False),
        _linear8("linear8_ffn_down", 32760, 13824, 5120, "none", True, 1, True),
    ]


# ------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A channel count: mostly a multiple of 8, not always."""
    n = _log_int(rng, lo, hi)
    return max(lo, n // 8 * 8) if rng.random() < 0.75 else n


def _draw_norm(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    most = _MAX_NORM * 2 // _BYTES[dtype]
    if rng.random() < 0.3:      # heads
        heads, C = rng.choice([1, 2, 3, 5, 10, 12, 14, 40]), rng.choice([32, 64, 72, 80, 96, 128, 128, 128, 160])
        rows = min(_log_int(rng, 1, 118800), most // (3 * heads * C))
        return {"kind": "norm", "rows": rows, "heads": heads, "C": C, "residual": False, "out": "same", "dtype": dtype,
                "fused": rng.random() < 0.7, "rowsum": False}
    C = _width(rng, 64, 16384)
    out = rng.choice(["same", "codes", "codes"])
    rows = min(_log_int(rng, 1, 118800), most // C)
    return {"kind": "norm", "rows": rows, "heads": 0, "C": C, "residual": rng.random() < 0.6, "out": out, "dtype": dtype,
            "fused": False, "rowsum": out == "codes" and rng.random() < 0.3}


def _draw_quant(rng):
    dtype, up = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.random() < 0.4
    C = _width(rng, 64, 16384)
    rows = min(_log_int(rng, 1, 118800), _MAX_QUANT * 2 // (_BYTES[dtype] * C * (2 if up else 1)))
    return {"kind": "quant", "rows": rows, "C": C, "act": rng.choice(["silu", "gelu_tanh", "gelu"] if up else ["none", "none", "gelu_tanh", "gelu"]),
            "up": up, "dtype": dtype}


def _draw_linear8(rng):
    M = _log_int(rng, 1, 118800)
    N, K = _width(rng, 64, 13824), _width(rng, 64, 13824)
    M = max(1, min(M, _MAX_FLOPS // (2 * K * N), _MAX_X // K, _MAX_Y // N))
    gate = rng.choice([0, 0, 1, 2])
    if gate:
        M = max(gate, M // gate * gate)
    return {"kind": "linear8", "M": M, "K": K, "N": N, "act": rng.choice(["none", "none", "gelu_tanh", "gelu", "silu"]),
            "bias": rng.random() < 0.7, "gate": gate, "residual": rng.random() < 0.5, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"])}


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    kind = rng.choices(["norm", "quant", "linear8"], [4, 3, 5])[0]
    return {"norm": _draw_norm, "quant": _draw_quant, "linear8": _draw_linear8}[kind](rng)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _tokens(g, M, K):
    """Tokens of varying magnitude with a few large channels, in 32 bits."""
    x = torch.randn((M, K), generator=g, device=DEV, dtype=torch.float32)
    x.mul_(torch.exp(0.3 * torch.randn((M, 1), generator=g, device=DEV)))
    x[:, torch.randperm(K, generator=g, device=DEV)[:max(1, K // 100)]] *= 8.0
    return x


def _norm_inputs(g, case):
    rows, heads, C, dt = case["rows"], case["heads"], case["C"], _DTYPES[case["dtype"]]
    if heads:
        x = _randn(g, (rows, heads * (3 if case["fused"] else 1), C), dt)[:, :heads]
    else:
        x = _tokens(g, rows, C).to(dt)
    return {"x": x, "w": (1.0 + _randn(g, (C,), torch.float32, 0.2)).to(dt),
            "residual": _randn(g, tuple(x.shape), dt, 2.0) if case["residual"] else None}


def _quant_inputs(g, case):
    rows, C, dt = case["rows"], case["C"], _DTYPES[case["dtype"]]
    if case["up"]:       # one product's output: the activation's argument and the factor, side by side
        both = _tokens(g, rows, 2 * C).to(dt)
        return {"x": both[:, :C], "up": both[:, C:]}
    return {"x": _tokens(g, rows, C).to(dt), "up": None}


def _codes(x):
    scale = x.abs().amax(1).div_(127.0)
    return x.div_(scale[:, None]).round_().to(torch.int8), scale


def _linear8_inputs(g, case):
    M, K, N, dt = case["M"], case["K"], case["N"], _DTYPES[case["dtype"]]
    codes, x_scale = _codes(_tokens(g, M, K))
    w, w_scale = _codes(_randn(g, (N, K), torch.float32, 1.0 / math.sqrt(K)))
    return {
        "codes": codes, "x_scale": x_scale, "w": w, "w_scale": w_scale,
        "b": _randn(g, (N,), dt, 0.1) if case["bias"] else None,
        "gate": _randn(g, (case["gate"], N), dt, 0.5) if case["gate"] else None,
        "residual": _randn(g, (M, N), dt) if case["residual"] else None,
    }


def prepare(case, seed):
    """What the caller's program holds before the call: this step's activations, the weights and, for the library's calls, the
    workspace it keeps."""
    g = _gen(seed)
    s = {"norm": _norm_inputs, "quant": _quant_inputs, "linear8": _linear8_inputs}[case["kind"]](g, case)
    s["case"] = case
    if own:
        import paper_2505_18663_amd as dvdq
        n = dvdq.linear8_workspace_bytes(case["M"], case["N"], case["K"]) if case["kind"] == "linear8" else 0
        s["workspace"] = torch.empty((n,), dtype=torch.uint8, device=DEV) if n else None
    return s


# ------------------------------------------------------------------ plain forms
_EPS = 1e-6


def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(z * -0.7071067811865476)
    if act == "gelu_tanh":
        return z * torch.sigmoid(1.5957691216057308 * (z + 0.044715 * z * z * z))
    return z


def _values(z, factor):
    """(values, codes) of rows z in 64 bits: codes = 127 z / max|z|, to the nearest, ties to the even one; the scale is factor * max|z| / 127."""
    top = z.abs().amax(-1, keepdim=True)
    codes = torch.round(127.0 * z / torch.where(top > 0, top, 1.0))
    return codes.float() * (factor * top / 127.0).float(), codes


def _plain_norm(s):
    c, x = s["case"], s["x"]
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    f = h.float()
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + _EPS)
    out = [] if s["residual"] is None else [h]
    if c["out"] == "same":
        return [(f * r * s["w"].float()).to(x.dtype)] + out
    values, codes = _values(h.double() * s["w"].double(), r.double())
    return [values] + ([codes.sum(-1).to(torch.int32)] if c["rowsum"] else []) + out


def _plain_quant(s):
    z = _act(s["x"].double(), s["case"]["act"])
    if s["up"] is not None:
        z = z * s["up"].double()
    return _values(z, 1.0)[0]


def _plain_linear8(s):
    z = (s["codes"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    if s["b"] is not None:
        z = z + s["b"].float()
    # (in 64 bits: 1 + tanh and 1 + erf have no digits left below zero otherwise)
    z = _act(z.double(), s["case"]["act"]).float() if s["case"]["act"] != "none" else z
    if s["gate"] is not None:
        z = (z.view(s["gate"].shape[0], -1, z.shape[1]) * s["gate"].float()[:, None]).view_as(z)
    if s["residual"] is not None:
        z = z + s["residual"].float()
    return z.to(_DTYPES[s["case"]["dtype"]])


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if not own:
        return {"norm": _plain_norm, "quant": _plain_quant, "linear8": _plain_linear8}[c["kind"]](s)
    import paper_2505_18663_amd as dvdq
    act = {"none": dvdq.ACT_NONE, "silu": dvdq.ACT_SILU, "gelu_tanh": dvdq.ACT_GELU_TANH, "gelu": dvdq.ACT_GELU}
    if c["kind"] == "linear8":
        return dvdq.linear8(s["codes"], s["x_scale"], s["w"], s["w_scale"], bias=s["b"], act=act[c["act"]], gate=s["gate"],
                            residual=s["residual"], dtype=_DTYPES[c["dtype"]], workspace=s["workspace"])
    if c["kind"] == "quant":
        codes, scale = dvdq.quant8(s["x"], up=s["up"], act=act[c["act"]])
        return codes * scale[:, None]
    if c["out"] == "same":
        out = dvdq.rms_norm(s["x"], s["w"], residual=s["residual"], eps=_EPS)
        return [out] if s["residual"] is None else list(out)
    codes, scale, *more = dvdq.rms_norm_quant(s["x"], s["w"], residual=s["residual"], eps=_EPS, want_rowsum=c["rowsum"])
    return [codes * scale[:, None]] + more


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = _BYTES[case["dtype"]]
    if case["kind"] == "linear8":
        M, K, N = case["M"], case["K"], case["N"]
        vec = (1 if case["bias"] else 0) + case["gate"]
        return {"bytes": M * K + N * K + 4 * (M + N) + e * (vec * N + M * N * (2 if case["residual"] else 1)), "flops": 2 * M * K * N}
    if case["kind"] == "quant":     # in once, a code and a scale out, and the values that the codes stand for
        n = case["rows"] * case["C"]
        return {"bytes": n * (e * (2 if case["up"] else 1) + 1 + 4) + 4 * case["rows"], "flops": n * (16 if case["act"] != "none" else 4)}
    rows = case["rows"] * max(1, case["heads"])
    n = rows * case["C"]
    out = e if case["out"] == "same" else 1 + 4
    return {"bytes": n * (e * (3 if case["residual"] else 1) + out) + e * case["C"] + (4 * rows if case["out"] == "codes" else 0),
            "flops": n * (8 if case["out"] == "codes" else 4)}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_codes(z):
    """The whole number next to 127 |z| / max|z|, by comparing 254 |z| with the odd multiples of the maximum; its sign; the maximum."""
    a = z.abs()
    top, _ = a.max(-1, keepdim=True)
    low = torch.floor(a * 127 / top.clamp(min=torch.finfo(torch.float64).tiny)).clamp(0, 126)
    over = 254 * a - (2 * low + 1) * top
    n = torch.where((over > 0) | ((over == 0) & (low % 2 == 1)), low + 1, low)
    return n * torch.sign(z), top


def _exact_act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def _in_parts(rows, columns, one):
    """one(first row, last row) -> a list of tensors, over parts of the rows that fit beside the inputs, joined"""
    step = max(1, (1 << 28) // columns)
    parts = [one(m, min(rows, m + step)) for m in range(0, rows, step)]
    return [torch.cat(p) for p in zip(*parts)]


def _exact_norm(case, s):
    w = s["w"].double()

    def one(a, b):
        h = s["x"][a:b].double()
        out = []
        if case["residual"]:
            h = (h + s["residual"][a:b].double()).to(s["x"].dtype).double()
            out = [h]
        root = torch.sqrt(torch.linalg.vector_norm(h, dim=-1, keepdim=True).square() / case["C"] + _EPS)
        if case["out"] == "same":
            return [h / root * w] + out
        n, top = _exact_codes(h * w)
        return [n * top / (127 * root)] + ([n.sum(-1).to(torch.int32)] if case["rowsum"] else []) + out

    return _in_parts(case["rows"], case["C"] * max(1, case["heads"]), one)


def _exact_quant(case, s):
    def one(a, b):
        z = _exact_act(s["x"][a:b].double(), case["act"])
        if case["up"]:
            z = z * s["up"][a:b].double()
        n, top = _exact_codes(z)
        return [n * (top / 127)]

    return _in_parts(case["rows"], case["C"], one)[0]


def _exact_linear8(case, s):
    w = (s["w"].double() * s["w_scale"].double()[:, None]).t().contiguous()
    per = case["M"] // case["gate"] if case["gate"] else 0

    def one(a, b):
        z = torch.matmul(s["codes"][a:b].double() * s["x_scale"][a:b].double()[:, None], w)
        if case["bias"]:
            z += s["b"].double()
        z = _exact_act(z, case["act"])
        if per:
            z *= s["gate"].double()[torch.arange(a, b, device=z.device) // per]
        if case["residual"]:
            z += s["residual"][a:b].double()
        return [z]

    return _in_parts(case["M"], max(case["N"], case["K"]), one)[0]


def exact(case, seed):
    """What `run` returns for these inputs, in 64 bits."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "quant": _exact_quant, "linear8": _exact_linear8}[case["kind"]](case, s)
