"""Timed cases of linear layers in 8 bits: activations and weights to 8 bits and back, the product of 8-bit integers with a scale per
token and per output channel, and its two gradients, which read the 8-bit weight and the 8-bit activations that were kept.

A case is one call of one of them, at a size that a model of this repository's parameter sets (or one like them) has.  `run`
computes it with elementary torch operations, or, where `own` is true, with this library's entry points.
"""
import math

import torch

own = False

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
TOP = {"int8": 127, "e4m3": 448}
LEAST = 2.0**-126
MOST_PRODUCT = 8192 * 14336 * 4096      # tokens x output x input features of the largest product
MOST_ELEMS = 8192 * 14336               # elements of the largest matrix that is taken to 8 bits and back


def _quant(**kw):
    """type: of the matrix in 16 or 32 bits.  code, group, pow2: form of the codes, columns per scale (0: the whole row), whether
    scales are powers of two.  pad: extra elements between two rows of that matrix."""
    case = dict(op="quant", rows=8192, cols=4096, type="bf16", code="int8", group=0, pow2=False, pad=0)
    case.update(kw)
    return case


def _linear(**kw):
    """tokens, out, inn: x8 [tokens, inn], w8 [out, inn], y and dy [tokens, out].  code, group, pow2: of x8, as above.  type: of
    what is computed.  pad: extra elements between two rows of x8, w8 and of y or dy.  add: the weight's gradient is added to what is there."""
    case = dict(op="linear", tokens=2048, out=4096, inn=4096, type="bf16", code="int8", group=0, pow2=False, pad=0)
    case.update(kw)
    if case["op"] == "weight_grad":
        case = dict(dict(add=False), **case)
    return case


def listed():
    return [
        # one decoded token of the 8B shapes, on its way into a product of 8-bit integers
        _quant(name="quant 1 x 4096", rows=1),
        # an MLP matrix of the 8B shapes after an optimizer step: a scale per output channel
        _quant(name="quant 14336 x 4096", rows=14336),
        # the inner activations of an MLP of the 8B shapes, kept for the backward pass: scales that are powers of two
        _quant(name="quant 8192 x 14336 /128", cols=14336, group=128, pow2=True),
        # a small fp32 model whose width is not a multiple of anything: kept activations back in 32 bits
        _quant(name="dequant 333 x 1001 e4m3 /128", op="dequant", rows=333, cols=1001, type="f32", code="e4m3", group=128, pow2=True),
        # kept activations of the 8B shapes back in 16 bits, for an operator that does not read codes
        _quant(name="dequant 8192 x 14336 /128", op="dequant", cols=14336, group=128, pow2=True),
        # one decoded token through an MLP matrix of the 8B shapes: one pass over the weight
        _linear(name="linear 1 x 14336 x 4096", tokens=1, out=14336),
        # two sequences of 1024 through the first MLP matrix of the 1.5B model
        _linear(name="linear 2048 x 6400 x 1600", out=6400, inn=1600),
        # a training step of the 8B shapes, eight sequences of 1024
        _linear(name="linear 8192 x 14336 x 4096", tokens=8192, out=14336),
        # a ragged batch through the 350M model's MLP
        _linear(name="input grad 1000 x 2736 x 1024", op="input_grad", tokens=1000, out=2736, inn=1024),
        # the gradient of the training step above
        _linear(name="input grad 8192 x 14336 x 4096", op="input_grad", tokens=8192, out=14336),
        # debugging a training loop of the 60M model: gradients in fp32, a ragged batch
        _linear(name="weight grad 777 x 1376 x 512 f32", op="weight_grad", tokens=777, out=1376, inn=512, type="f32", code="e4m3", group=128, pow2=True),
        # the training step above, from activations with a scale per 128 columns
        _linear(name="weight grad 8192 x 14336 x 4096", op="weight_grad", tokens=8192, out=14336, group=128, pow2=True),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "dequant", "linear", "input_grad", "weight_grad"])
    code = rng.choice(["int8", "int8", "e4m3"])
    form = dict(code=code, group=rng.choice([0, 128]), pow2=code == "e4m3" or rng.random() < 0.5)
    if op in ("quant", "dequant"):
        rows, cols = _spread(rng, 1, 65536), _spread(rng, 64, 32768)
        cols = cols if rng.random() < 0.3 else max(64, cols // 8 * 8)
        rows = max(1, min(rows, MOST_ELEMS // cols))
        return _quant(op=op, rows=rows, cols=cols, type=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 8, 5]), **form)
    tokens, out, inn = _spread(rng, 1, 16384), 8 * _spread(rng, 8, 1792), 8 * _spread(rng, 8, 1792)
    tokens = max(1, min(tokens, MOST_PRODUCT // (out * inn)))
    case = dict(op=op, tokens=tokens, out=out, inn=inn, type=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 64]))
    if op != "weight_grad":
        return _linear(**case)
    if case["type"] == "f32":
        form["pow2"] = True             # (other scales are for gradients in 16 bits: the decoded numbers are rounded to that)
    return _linear(add=rng.random() < 0.3, **case, **form)


# ---------------------------------------------------------------------------------------------- inputs

def _pitched(x, pad, unit=1):
    """The same matrix, its rows `pad` elements further apart than they are long (and a multiple of `unit`)."""
    rows, cols = x.shape
    ld = -(-(cols + pad) // unit) * unit
    if ld == cols:
        return x
    wide = torch.zeros(rows, ld, dtype=x.dtype, device=x.device)
    wide[:, :cols] = x
    return wide[:, :cols]


def _activations(gen, rows, cols):
    """Hidden states behind a norm: a few columns are much larger than the others, and tokens differ in size."""
    columns = 1 + 15 * (torch.rand(cols, generator=gen, device="cuda") < 0.004)
    sizes = 0.5 + torch.rand(rows, 1, generator=gen, device="cuda")
    return torch.randn(rows, cols, generator=gen, device="cuda") * columns * sizes


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case, "kept": {}}
    if case["op"] in ("quant", "dequant"):
        x = _activations(gen, case["rows"], case["cols"]).to(TYPES[case["type"]])
        if case["op"] == "quant":
            state["x"] = _pitched(x, case["pad"])
        else:
            state["codes"], state["scales"] = _to_codes(x, case)
        return state
    tokens, out, inn = case["tokens"], case["out"], case["inn"]
    if case["op"] != "weight_grad":
        weight = torch.randn(out, inn, generator=gen, device="cuda") * 0.02 * (0.5 + torch.rand(out, 1, generator=gen, device="cuda"))
        w8, state["ws"] = _to_codes(weight.to(BF16), _quant(rows=out, cols=inn))
        state["w8"] = _pitched(w8, case["pad"], 16)
    if case["op"] != "input_grad":
        x8, state["xs"] = _to_codes(_activations(gen, tokens, inn).to(BF16), dict(case, rows=tokens, cols=inn))
        state["x8"] = _pitched(x8, case["pad"], 16)
    if case["op"] != "linear":
        state["dy"] = _pitched((1e-3 * torch.randn(tokens, out, generator=gen, device="cuda")).to(BF16), case["pad"], 8)
    if case["op"] == "weight_grad" and case["add"]:
        state["before"] = (1e-2 * torch.randn(out, inn, generator=gen, device="cuda")).to(TYPES[case["type"]])
    return state


# ---------------------------------------------------------------------------------------------- plain forms

def _to_codes(x, case):
    """Codes and scales of a matrix, in groups of columns."""
    rows, cols = x.shape
    group, top = case["group"] or cols, TOP[case["code"]]
    n = -(-cols // group)
    parts = torch.nn.functional.pad(x.float(), (0, n * group - cols)).view(rows, n, group)
    most = parts.abs().amax(2, keepdim=True)
    if case["pow2"]:
        fraction, power = torch.frexp(most)                   # most = fraction 2^power, fraction in [1/2, 1)
        limit, limit_power = math.frexp(top)
        power = torch.where(fraction > limit, power + 1, power) - limit_power
        scale = torch.ldexp(torch.ones_like(most, dtype=torch.float64), power.clamp(min=-126)).float()
    else:
        scale = (most.double() / top).float().clamp(min=LEAST)
    scale = torch.where(most > 0, scale, 1.0)
    # the quotient in 64 bits: next to half a step, its rounding to 32 would decide which way a code goes
    codes = torch.empty(rows, n * group, dtype=torch.int8 if case["code"] == "int8" else E4M3, device=x.device)
    for i in range(0, rows, 2048):
        quotient = (parts[i:i + 2048].double() / scale[i:i + 2048].double()).view(-1, n * group)
        codes[i:i + 2048] = quotient.round().to(torch.int8) if case["code"] == "int8" else quotient.float().to(E4M3)
    return codes[:, :cols].contiguous(), scale[:, :, 0]


def _decoded(codes, scales):
    """codes times their scales in 32 bits; scales: one per row, or per 128 columns of it."""
    wide = codes.float()
    cols = codes.shape[1]
    return wide * (scales if scales.shape[1] == 1 else scales.repeat_interleave(128, 1)[:, :cols])


def _plain_quant(state):
    codes, scales = _to_codes(state["x"], state["case"])
    return {"codes": codes, "scales": scales}


def _plain_dequant(state):
    return {"x": _decoded(state["codes"], state["scales"]).to(TYPES[state["case"]["type"]])}


def _plain_linear(state):
    sums = state["x8"].float() @ state["w8"].float().T        # whole numbers, far below 2^24
    return {"y": (sums * state["xs"] * state["ws"].T).to(TYPES[state["case"]["type"]])}


def _plain_input_grad(state):
    return {"dx": (state["dy"].float() @ _decoded(state["w8"], state["ws"])).to(TYPES[state["case"]["type"]])}


def _plain_weight_grad(state):
    dw = state["dy"].float().T @ _decoded(state["x8"], state["xs"])
    if "before" in state:
        dw = dw + state["before"].float()
    return {"dweight": dw.to(TYPES[state["case"]["type"]])}


# ---------------------------------------------------------------------------------------------- the library's calls

def _type_of(A, case):
    return A.TYPE_F32 if case["type"] == "f32" else A.TYPE_BF16


def _code_of(A, case):
    return A.CODE_E4M3 if case["code"] == "e4m3" else A.CODE_INT8


def _own_quant(state):
    import paper_2510_09103_b200 as A
    k, case = state["kept"], state["case"]
    if not k:                           # the descriptor and the outputs that a program keeps from one call to the next
        rows, cols = case["rows"], case["cols"]
        k["desc"] = A.quant8_desc(rows, cols, dtype=_type_of(A, case), code=_code_of(A, case), group=case["group"], pow2=case["pow2"],
                                  x_ld=cols + case["pad"])
        if case["op"] == "quant":
            k["codes"] = torch.empty(rows, cols, dtype=E4M3 if case["code"] == "e4m3" else torch.int8, device="cuda")
            k["scales"] = torch.empty(rows, -(-cols // (case["group"] or cols)), device="cuda")
        else:
            k["x"] = torch.empty_strided((rows, cols), (cols + case["pad"], 1), dtype=TYPES[case["type"]], device="cuda")
    if case["op"] == "quant":
        A.adapm_quant8(k["desc"], state["x"], k["codes"], k["scales"])
        return {"codes": k["codes"], "scales": k["scales"]}
    A.adapm_dequant8(k["desc"], state["codes"], state["scales"], k["x"])
    return {"x": k["x"]}


def _own_product(state):
    import paper_2510_09103_b200 as A
    k, case = state["kept"], state["case"]
    op, tokens, out, inn = case["op"], case["tokens"], case["out"], case["inn"]
    if not k:                           # the descriptor, scratch and outputs that a program keeps from one call to the next
        of_8 = state["w8"] if "w8" in state else state["x8"]
        rows, cols = {"linear": (tokens, out), "input_grad": (tokens, inn), "weight_grad": (out, inn)}[op]
        y_ld = state["dy"].stride(0) if "dy" in state else out + case["pad"]
        k["desc"] = A.linear8_desc(tokens, out, inn, x_code=_code_of(A, case), x_group=case["group"], y_dtype=_type_of(A, case),
                                   dx_dtype=_type_of(A, case), dweight_dtype=_type_of(A, case), accumulate=case.get("add", False),
                                   x8_ld=of_8.stride(0), w8_ld=of_8.stride(0), y_ld=y_ld)
        which = {"linear": A.LINEAR8_FORWARD, "input_grad": A.LINEAR8_INPUT_GRAD, "weight_grad": A.LINEAR8_WEIGHT_GRAD}[op]
        k["scratch"] = torch.empty(A.adapm_linear8_scratch_bytes(k["desc"], which), dtype=torch.uint8, device="cuda")
        k["out"] = torch.empty_strided((rows, cols), (y_ld if op == "linear" else cols, 1), dtype=TYPES[case["type"]], device="cuda")
    if op == "linear":
        A.adapm_linear8_forward(k["desc"], state["x8"], state["xs"], state["w8"], state["ws"], k["out"], k["scratch"])
        return {"y": k["out"]}
    if op == "input_grad":
        A.adapm_linear8_input_grad(k["desc"], state["dy"], state["w8"], state["ws"], k["out"], k["scratch"])
        return {"dx": k["out"]}
    if case["add"]:
        k["out"].copy_(state["before"])
    A.adapm_linear8_weight_grad(k["desc"], state["dy"], state["x8"], state["xs"], k["out"], k["scratch"])
    return {"dweight": k["out"]}


PLAIN = {"quant": _plain_quant, "dequant": _plain_dequant, "linear": _plain_linear, "input_grad": _plain_input_grad, "weight_grad": _plain_weight_grad}
OWN = {"quant": _own_quant, "dequant": _own_quant, "linear": _own_product, "input_grad": _own_product, "weight_grad": _own_product}


def run(state):
    op = state["case"]["op"]
    return OWN[op](state) if own else PLAIN[op](state)


def work(case):
    size = {"bf16": 2, "f32": 4}[case["type"]]
    if case["op"] in ("quant", "dequant"):
        scales = case["rows"] * (-(-case["cols"] // (case["group"] or case["cols"])))
        return {"bytes": case["rows"] * case["cols"] * (size + 1) + 4 * scales, "flops": 0}
    tokens, out, inn = case["tokens"], case["out"], case["inn"]
    flops = 2.0 * tokens * out * inn
    if case["op"] == "linear":
        return {"bytes": (tokens + out) * (inn + 4) + size * tokens * out, "flops": flops}
    if case["op"] == "input_grad":
        return {"bytes": 2 * tokens * out + out * (inn + 4) + size * tokens * inn, "flops": flops}
    scales = tokens * (-(-inn // (case["group"] or inn)))
    return {"bytes": 2 * tokens * out + tokens * inn + 4 * scales + size * out * inn * (2 if case["add"] else 1), "flops": flops}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits

def _exact_quant(state):
    case, x = state["case"], state["x"].double()
    group, top = case["group"] or case["cols"], 127.0 if case["code"] == "int8" else 448.0
    codes, scales = [], []
    for part in x.split(group, 1):
        m = part.abs().max(1, keepdim=True).values
        if case["pow2"]:
            # the least power of two whose product with the greatest code reaches m: from above, halved while half of it does too
            s = torch.exp2(torch.ceil(torch.log2(m.clamp(min=1e-300) / top)) + 1)
            for _ in range(3):
                s = torch.where(s / 2 * top >= m, s / 2, s)
            s = s.clamp(min=2.0**-126)
        else:
            s = (m / top).float().double().clamp(min=2.0**-126)      # held in 32 bits
        s = torch.where(m == 0, 1.0, s)
        scales.append(s)
        codes.append(torch.round(part / s).to(torch.int8) if case["code"] == "int8" else part / s)
    return {"codes": torch.cat(codes, 1), "scales": torch.cat(scales, 1)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quant":
        return _exact_quant(state)
    if case["op"] == "dequant":
        scales = state["scales"].double()
        column = torch.arange(case["cols"], device="cuda") // (case["group"] or case["cols"])
        return {"x": state["codes"].double() * scales[:, column]}
    if case["op"] == "linear":
        y = torch.einsum("tk,nk->tn", state["x8"].double(), state["w8"].double())
        return {"y": torch.einsum("tn,t,n->tn", y, state["xs"][:, 0].double(), state["ws"][:, 0].double())}
    dy = state["dy"].double()
    if case["op"] == "input_grad":
        return {"dx": torch.einsum("tn,nk->tk", dy * state["ws"][:, 0].double(), state["w8"].double())}
    group = case["group"] or case["inn"]
    parts = [torch.einsum("tn,tk->nk", dy * state["xs"][:, i:i + 1].double(), x8.double()) for i, x8 in enumerate(state["x8"].split(group, 1))]
    dw = torch.cat(parts, 1)
    return {"dweight": dw + state["before"].double() if "before" in state else dw}
