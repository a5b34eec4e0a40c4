"""What the dense half of a decoder layer costs in 8 bits: the norm that adds the residual and leaves e4m3 codes, the product
of such codes with 8-bit weights, and the gated feed-forward block, each with its plain form in PyTorch.

``listed()`` are the measured cases, ``draw()`` gives more of the same ranges.  ``run()`` makes one pass: with ``own`` the
calls a user makes of the package, otherwise the plain form.  Sizes are generic ones of decoders.

8-bit rows are e4m3 codes ``[batch, tokens, features]`` with a float32 scale for every row and block of 128 features, stored
``[block][row]``; 8-bit weights are e4m3 codes ``[out, in]`` with a float32 scale for every block of 128 by 128.  A code
stands for itself times its scale.  A block of rows whose largest magnitude is m (at least 2^-60) has the scale m / 448.
"""
import math

import torch

own = False

BLOCK = 128
LARGEST = 448.0                              # the largest e4m3 number
LEAST = 2.0 ** -60                           # blocks of smaller values share this magnitude
EPS = 1e-6


def listed():
    return [
        # one new token of one conversation enters a layer: a launch's latency
        dict(name="norm_one_token", op="norm", dtype="bf16", batch=1, tokens=1, width=4096, norm=True, res=True),
        # prompts of several conversations, the residual stream read and written
        dict(name="norm_prompts", op="norm", dtype="bf16", batch=3, tokens=1367, width=4096, norm=True, res=True),
        # the first norm of a network in fp32: nothing to add, a width that ends inside a block
        dict(name="norm_f32_first", op="norm", dtype="f32", batch=2, tokens=509, width=5008, norm=True, res=False),
        # the context of an attention on its way into the projection behind it: codes of the values as they are
        dict(name="codes_of_context", op="norm", dtype="bf16", batch=8, tokens=1024, width=8192, norm=False, res=False),
        # one token's queries, keys and values: latency and the weights' way from memory
        dict(name="gemm_one_token", op="gemm", dtype="bf16", batch=1, tokens=1, cin=4096, cout=6144, bias=False, res=False, act="none"),
        # a decoding step of a full server through the projection back to the residual stream
        dict(name="gemm_step", op="gemm", dtype="bf16", batch=64, tokens=1, cin=14336, cout=4096, bias=False, res=True, act="none"),
        # a few prompts in fp32: odd extents, the inner one ends inside a block
        dict(name="gemm_f32_odd", op="gemm", dtype="f32", batch=3, tokens=111, cin=2000, cout=1111, bias=True, res=False, act="gelu"),
        # many long prompts of a wide decoder
        dict(name="gemm_large", op="gemm", dtype="bf16", batch=8, tokens=1024, cin=8192, cout=8192, bias=False, res=False, act="none"),
        # one token through a feed-forward block's first half
        dict(name="gated_one_token", op="gated", dtype="bf16", batch=1, tokens=1, cin=4096, cout=14336, act="silu", codes=True),
        # a decoding step of many conversations
        dict(name="gated_step", op="gated", dtype="bf16", batch=48, tokens=1, cin=5120, cout=13824, act="silu", codes=True),
        # a long prompt
        dict(name="gated_prompt", op="gated", dtype="bf16", batch=1, tokens=4096, cin=4096, cout=14336, act="silu", codes=True),
        # short prompts, odd extents, the result in the tenant's type
        dict(name="gated_odd", op="gated", dtype="bf16", batch=3, tokens=259, cin=2064, cout=5520, act="gelu_tanh", codes=False),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _rows(rng, most):
    rows = _log(rng, 1, most)
    tokens = 1 if rng.random() < 0.4 else min(rows, _log(rng, 1, 1500))
    return dict(batch=max(1, rows // tokens), tokens=tokens)


def draw(rng):
    op = rng.choice(("norm", "gemm", "gemm", "gated", "gated"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        norm = rng.choice((True, True, False))
        width = 16 * _log(rng, 16, 1024)
        return dict(op=op, dtype=dtype, width=width, norm=norm, res=rng.choice((False, True)), **_rows(rng, min(16384, 2 ** 24 // width)))
    cin = 16 * _log(rng, 16, 1024)
    if op == "gemm":
        cout = rng.choice((_log(rng, 100, 20000), 16 * _log(rng, 8, 1024)))
        act = rng.choice(("none", "none", "relu", "gelu"))
        return dict(op=op, dtype=dtype, cin=cin, cout=cout, bias=rng.choice((False, True)), res=rng.choice((False, True)), act=act,
                    **_rows(rng, min(8192, 2 ** 38 // (cin * cout))))
    cout = 16 * _log(rng, 16, 1024)
    return dict(op=op, dtype=dtype, cin=cin, cout=cout, act=rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu")), codes=rng.choice((True, True, False)),
                **_rows(rng, min(8192, 2 ** 37 // (cin * cout))))


# -- what a program has in hand ---------------------------------------------------------------------------------------------

def _in_blocks(x):
    """x [..., n] as [..., blocks, 128], zeros behind the end."""
    n = x.shape[-1]
    pad = -n % BLOCK
    if pad:
        x = torch.cat((x, x.new_zeros(*x.shape[:-1], pad)), -1)
    return x.reshape(*x.shape[:-1], -1, BLOCK)


def _codes(x):
    """Rows x [rows, n] in 32 bits as e4m3 codes [rows, n] and scales [blocks, rows]."""
    y = _in_blocks(x)
    m = y.abs().amax(-1, keepdim=True).clamp_min(LEAST)
    codes = (y * (LARGEST / m)).to(torch.float8_e4m3fn)
    return codes.reshape(x.shape[0], -1)[:, :x.shape[1]].contiguous(), (m / LARGEST)[..., 0].t().contiguous()


def _weight(x):
    """Weights x [out, in] in 32 bits as e4m3 codes and scales of blocks of 128 by 128."""
    out, cin = x.shape
    y = _in_blocks(x)
    pad = -out % BLOCK
    if pad:
        y = torch.cat((y, y.new_zeros(pad, *y.shape[1:])), 0)
    y = y.reshape(-1, BLOCK, y.shape[1], BLOCK)
    m = y.abs().amax((1, 3), keepdim=True).clamp_min(LEAST)
    codes = (y * (LARGEST / m)).to(torch.float8_e4m3fn).reshape(out + pad, -1)[:out, :cin].contiguous()
    return codes, (m / LARGEST)[:, 0, :, 0].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n, t = case["batch"], case["tokens"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def stream(width):
        """A residual stream: a few features are much larger than the rest."""
        return (normal(n, t, width) * (1.0 + 8.0 * (normal(width).abs() > 2.5))).to(dtype)

    def out_rows(width):
        return (torch.empty((n, t, width), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((-(-width // BLOCK), n * t), device="cuda"))

    s = dict(case, dtype=dtype)
    if case["op"] == "norm":
        w = case["width"]
        s["x"] = stream(w)
        s["res_in"] = stream(w) if case["res"] else None
        s["sum"] = torch.empty_like(s["x"]) if case["res"] else None
        s["gamma"] = 1.0 + 0.2 * normal(w) if case["norm"] else None
        s["codes_out"], s["scales_out"] = out_rows(w)
        return s
    cin, cout = case["cin"], case["cout"]
    codes, s["scales"] = _codes(normal(n * t, cin) * (1.0 + 3.0 * (normal(cin).abs() > 2.5)))
    s["codes_in"] = codes.reshape(n, t, cin)
    if case["op"] == "gemm":
        s["weight"] = _weight(normal(cout, cin) * cin ** -0.5)
        s["bias_in"] = normal(cout) if case["bias"] else None
        s["res_in"] = normal(n, t, cout).to(dtype) if case["res"] else None
        s["out"] = torch.empty((n, t, cout), dtype=dtype, device="cuda")
        return s
    s["gate"], s["up"] = (_weight(normal(cout, cin) * 1.5 * cin ** -0.5) for _ in range(2))
    if case["codes"]:
        s["codes_out"], s["scales_out"] = out_rows(cout)
    else:
        s["out"] = torch.empty((n, t, cout), dtype=dtype, device="cuda")
    return s


# -- one pass ---------------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm, "gemm": _gemm, "gated": _gated}[state["op"]](state)


def _run_own(s):
    if "session" not in s:                   # the loaded operator list: what a program keeps
        from paper_2304_11745_amd import tokens as T
        ops = T.OpList(s["dtype"], s["batch"])
        if s["op"] == "norm":
            rows = T.Fp8Rows(s["codes_out"], s["scales_out"])
            if s["norm"]:
                ops.rmsnorm_fp8(s["x"], rows, s["gamma"], eps=EPS, res=s["res_in"], sum=s["sum"])
            else:
                ops.quantise_fp8(s["x"], rows, res=s["res_in"], sum=s["sum"])
        elif s["op"] == "gemm":
            ops.gemm_fp8(T.Fp8Rows(s["codes_in"], s["scales"]), T.Fp8Weight(*s["weight"]), s["out"], bias=s["bias_in"], act=s["act"], res=s["res_in"])
        else:
            y = T.Fp8Rows(s["codes_out"], s["scales_out"]) if s["codes"] else s["out"]
            ops.gated_fp8(T.Fp8Rows(s["codes_in"], s["scales"]), T.Fp8Weight(*s["gate"]), T.Fp8Weight(*s["up"]), y, act=s["act"])
        s["session"] = T.TokenSession([ops])
    s["session"].enqueue(0)
    if s["op"] == "norm":
        return {"codes": s["codes_out"], "scales": s["scales_out"], "sum": s["sum"]}
    if s["op"] == "gated" and s["codes"]:
        return {"codes": s["codes_out"], "scales": s["scales_out"]}
    return s["out"]


def _norm(s):
    n, t, w = s["batch"], s["tokens"], s["width"]
    h = s["x"].float()
    if s["res"]:
        h = h + s["res_in"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["gamma"] if s["norm"] else h
    codes, scales = _codes(y.reshape(n * t, w))
    return {"codes": codes.reshape(n, t, w), "scales": scales, "sum": h.to(s["dtype"]) if s["res"] else None}


def _input(s):
    """The rows [batch * tokens, cin] that the codes stand for."""
    rows = s["codes_in"].float().reshape(-1, s["cin"])
    return rows * s["scales"].t().repeat_interleave(BLOCK, 1)[:, :s["cin"]]


def _weights(pair):
    codes, scales = pair
    return codes.float() * scales.repeat_interleave(BLOCK, 0)[:codes.shape[0]].repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _act(x, name):
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x.clamp_min(0.0) if name == "relu" else x


def _gemm(s):
    y = _input(s) @ _weights(s["weight"]).t()
    if s["bias"]:
        y = y + s["bias_in"]
    if s["res"]:
        y = y + s["res_in"].float().reshape(y.shape)
    return _act(y, s["act"]).to(s["dtype"]).reshape(s["batch"], s["tokens"], -1)


def _gated(s):
    x = _input(s)
    y = _act(x @ _weights(s["gate"]).t(), s["act"]) * (x @ _weights(s["up"]).t())
    if not s["codes"]:
        return y.to(s["dtype"]).reshape(s["batch"], s["tokens"], -1)
    codes, scales = _codes(y)
    return {"codes": codes.reshape(s["batch"], s["tokens"], -1), "scales": scales}


# -- the same from the definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    """Codes before their rounding: a row's values over their block's scale."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gemm": _exact_gemm, "gated": _exact_gated}[case["op"]](s)


def _exact_rows(y, n, t):
    rows, width = y.shape
    codes, scales = torch.empty_like(y), y.new_empty(-(-width // BLOCK), rows)
    for b in range(scales.shape[0]):
        part = y[:, b * BLOCK:(b + 1) * BLOCK]
        scales[b] = torch.maximum(part.max(1).values, -part.min(1).values).clamp_min(LEAST) / 448
        codes[:, b * BLOCK:(b + 1) * BLOCK] = part / scales[b][:, None]
    return {"codes": codes.reshape(n, t, width), "scales": scales}


def _exact_norm(s):
    n, t, w = s["batch"], s["tokens"], s["width"]
    h = s["x"].double().reshape(n * t, w)
    if s["res"]:
        h += s["res_in"].double().reshape(n * t, w)
    y = h
    if s["norm"]:
        y = h / ((h ** 2).sum(1, keepdim=True) / w + EPS).sqrt() * s["gamma"].double()
    out = _exact_rows(y, n, t)
    out["sum"] = h.reshape(n, t, w) if s["res"] else None
    return out


def _exact_product(s, weight):
    """Block by block of 128 inner features."""
    codes, scales = weight
    x = s["codes_in"].double().reshape(-1, s["cin"])
    of = torch.arange(codes.shape[0], device="cuda") // BLOCK
    y = x.new_zeros(x.shape[0], codes.shape[0])
    for b in range(scales.shape[1]):
        k = slice(b * BLOCK, (b + 1) * BLOCK)
        y += x[:, k].contiguous() @ codes[:, k].double().T.contiguous() * s["scales"][b].double()[:, None] * scales[of, b].double()
    return y


def _exact_act(x, name):
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * torch.special.ndtr(x)
    if name == "gelu_tanh":
        return x * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))
    return torch.relu(x) if name == "relu" else x


def _exact_gemm(s):
    y = _exact_product(s, s["weight"])
    for more in (s["bias_in"], s["res_in"]):
        if more is not None:
            y += more.double().reshape(-1, s["cout"])
    return _exact_act(y, s["act"]).reshape(s["batch"], s["tokens"], -1)


def _exact_gated(s):
    y = _exact_act(_exact_product(s, s["gate"]), s["act"]) * _exact_product(s, s["up"])
    if s["codes"]:
        return _exact_rows(y, s["batch"], s["tokens"])
    return y.reshape(s["batch"], s["tokens"], -1)


# -- what a pass cannot do without ------------------------------------------------------------------------------------------

def _row_bytes(rows, width):
    return rows * width + 4 * rows * -(-width // BLOCK)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    rows = case["batch"] * case["tokens"]
    if case["op"] == "norm":
        w = case["width"]
        return {"bytes": rows * w * e * (3 if case["res"] else 1) + _row_bytes(rows, w) + (4 * w if case["norm"] else 0), "flops": rows * w * (8 if case["norm"] else 3)}
    cin, cout = case["cin"], case["cout"]
    weights = cout * cin + 4 * -(-cout // BLOCK) * -(-cin // BLOCK)
    if case["op"] == "gemm":
        return {"bytes": _row_bytes(rows, cin) + weights + rows * cout * e * (2 if case["res"] else 1) + (4 * cout if case["bias"] else 0), "flops": 2 * rows * cout * cin}
    return {"bytes": _row_bytes(rows, cin) + 2 * weights + (_row_bytes(rows, cout) if case["codes"] else rows * cout * e), "flops": 4 * rows * cout * cin}
