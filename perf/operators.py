"""Timed cases of the operators at the end of a decoder's training step: the head's loss over the vocabulary and its
gradient, RMS normalisation with the residual's addition and its gradient, and dropout.

A case is one call of one of them, at a size that a model of this repository's parameter sets (or one like them) has.  `run`
computes it with elementary torch operations, or, where `own` is true, with this library's entry points.
"""
import math

import torch

own = False

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
IGNORE = -100
MOST_LOSS = 8192 * 128256 * 4096        # tokens x vocabulary x width of the largest case
MOST_ELEMS = 65536 * 1600               # elements of the largest elementwise case


def _loss(**kw):
    """tokens, vocab, width: of hidden [tokens, width] and weight [vocab, width].  pad: extra elements between two rows of
    hidden.  ignored: share of the tokens whose target is the ignored one.  smooth, z: label smoothing and the
    coefficient of lse^2.  grad only: dtype of dhidden and of dweight, whether every token has a weight of its own."""
    case = dict(op="loss", tokens=2048, vocab=50257, width=768, pad=0, ignored=0.0, smooth=0.0, z=0.0)
    case.update(kw)
    if case["op"] == "loss_grad":
        case = dict(dict(dhidden="bf16", dweight="bf16", weighted=False), **case)
    return case


def _norm(**kw):
    """residual, p: whether a residual is added, and the dropout of the branch before it.  q8: None, 0 (one scale per row)
    or 128 (one per 128 columns); with q8 the output is in 8 bits only.  weight: type of the norm's weight."""
    case = dict(op="norm", rows=8192, cols=1600, type="bf16", weight="bf16", residual=True, p=0.0, eps=1e-5)
    case.update(kw)
    if case["op"] == "norm":
        case = dict(dict(q8=None), **case)
    else:
        case = dict(dict(dweight="bf16"), **case)
    return case


def _dropout(**kw):
    case = dict(op="dropout", rows=8192, cols=1600, type="bf16", residual=False, p=0.1)
    case.update(kw)
    return case


def listed():
    return [
        # scoring the answer of one short request with the 60M model: launches and one pass over the head's weight
        _loss(name="loss 24 x 32000 x 512", tokens=24, vocab=32000, width=512),
        # validation loss of the 1.5B model on eight sequences of 1024
        _loss(name="loss 8192 x 50257 x 1600", tokens=8192, width=1600),
        # debugging a training loop: the two-layer model in fp32, every gradient in fp32
        _loss(name="grad 512 x 4096 x 256 f32", op="loss_grad", tokens=512, vocab=4096, width=256, dhidden="f32", dweight="f32"),
        # pre-training of the 1.5B model, eight sequences of 1024
        _loss(name="grad 8192 x 50257 x 1600", op="loss_grad", tokens=8192, width=1600, z=1e-4),
        # instruction tuning of the 8B shapes: half of the tokens are prompts, which are not trained on
        _loss(name="grad 8192 x 128256 x 4096", op="loss_grad", tokens=8192, vocab=128256, width=4096, ignored=0.5),
        # one decoded token of the 8B shapes, ready for a product in 8 bits
        _norm(name="norm 1 x 4096 8 bits", rows=1, cols=4096, q8=0),
        # pre-norm of the 1.5B model in training, the branch's dropout with it
        _norm(name="norm 16384 x 1600 dropout", rows=16384, cols=1600, p=0.1),
        # a prompt of the 8B shapes, output in 8 bits with a scale per 128 columns
        _norm(name="norm 8192 x 4096 8 bits/128", rows=8192, cols=4096, q8=128),
        # the gradient of the second of these
        _norm(name="norm grad 16384 x 1600", op="norm_grad", rows=16384, cols=1600, p=0.1),
        # a small fp32 model whose width is not a multiple of anything
        _norm(name="norm grad 333 x 1001 f32", op="norm_grad", rows=333, cols=1001, type="f32", weight="f32", dweight="f32"),
        # the embedding's dropout of the smallest model
        _dropout(name="dropout 1024 x 256", rows=1024, cols=256, p=0.1),
        # an attention output's dropout, added to the residual, sixty-four sequences of 1024
        _dropout(name="dropout 65536 x 1600", rows=65536, cols=1600, residual=True),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["loss", "loss_grad", "norm", "norm_grad", "dropout"])
    if op in ("loss", "loss_grad"):
        tokens, vocab, width = _spread(rng, 1, 8192), _spread(rng, 1000, 131072), 8 * _spread(rng, 8, 512)
        tokens = max(1, min(tokens, MOST_LOSS // (vocab * width)))
        case = _loss(op=op, tokens=tokens, vocab=vocab, width=width, pad=rng.choice([0, 0, 8, 64]),
                     ignored=rng.choice([0.0, 0.0, 0.1, 0.5, 0.9]), smooth=rng.choice([0.0, 0.0, 0.1]), z=rng.choice([0.0, 1e-4]))
        if op == "loss_grad":
            case.update(dhidden=rng.choice(["bf16", "f32"]), dweight=rng.choice(["bf16", "f32"]), weighted=rng.random() < 0.5)
        return case
    rows, cols = _spread(rng, 1, 65536), _spread(rng, 64, 16384)
    cols = cols if rng.random() < 0.3 else max(64, cols // 8 * 8)
    rows = max(1, min(rows, MOST_ELEMS // cols))
    kind = rng.choice(["bf16", "bf16", "f32"])
    p = rng.choice([0.0, 0.1, 0.3])
    if op == "dropout":
        return _dropout(rows=rows, cols=cols, type=kind, residual=rng.random() < 0.5, p=p or 0.5)
    case = _norm(op=op, rows=rows, cols=cols, type=kind, weight=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.7, p=p)
    if op == "norm":
        case.update(q8=rng.choice([None, None, 0, 128]))
    else:
        case.update(dweight=rng.choice(["bf16", "f32"]))
    return case


def _valid(case):
    return case["tokens"] - int(round(case["tokens"] * case["ignored"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    state = {"case": case, "kept": {}}
    if case["op"] in ("loss", "loss_grad"):
        tokens, vocab, width = case["tokens"], case["vocab"], case["width"]
        weight = (normal(vocab, width) * 0.02).to(BF16)
        targets = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
        # hidden states of a model in training: some targets are far up already, most are not
        toward = weight[targets].float()
        toward /= toward.square().sum(1, keepdim=True).sqrt()
        strength = 16 * torch.rand(tokens, 1, generator=gen, device="cuda") ** 2
        hidden = torch.zeros(tokens, width + case["pad"], dtype=BF16, device="cuda")
        hidden[:, :width] = (normal(tokens, width) + strength * toward).to(BF16)
        ignored = torch.randperm(tokens, generator=gen, device="cuda")[: tokens - _valid(case)]
        targets[ignored] = IGNORE
        state.update(hidden=hidden[:, :width], weight=weight, targets=targets)
        if case["op"] == "loss_grad":
            parts = [torch.logsumexp(h.float() @ weight.float().T, 1) for h in state["hidden"].split(4096)]
            state["lse"] = torch.cat(parts)
            state["scale"] = 1.0 / max(1, _valid(case))
            state["dloss"] = 0.5 + torch.rand(tokens, generator=gen, device="cuda") if case["weighted"] else None
        return state
    kind = TYPES[case["type"]]
    rows, cols = case["rows"], case["cols"]
    state["seed"], state["offset"] = 0x5EED0000 + seed, 3
    # the residual stream of a deep model: rows of different lengths, a few columns much larger than the others
    columns = 1 + 20 * (torch.rand(cols, generator=gen, device="cuda") < 0.004)
    stream = (normal(rows, cols) * columns * (0.5 + torch.rand(rows, 1, generator=gen, device="cuda"))).to(kind)
    if case["op"] == "dropout":
        state.update(x=normal(rows, cols).to(kind), residual=stream if case["residual"] else None)
        return state
    state["weight"] = (1 + 0.1 * normal(cols)).to(TYPES[case["weight"]])
    if case["op"] == "norm":
        alone = not case["residual"]
        state.update(x=stream if alone else normal(rows, cols).to(kind), residual=None if alone else stream)
    else:
        state.update(sum=stream, rstd=(stream.float().square().mean(1) + case["eps"]).rsqrt(), dy=(1e-3 * normal(rows, cols)).to(kind),
                     dsum=(1e-3 * normal(rows, cols)).to(kind) if case["residual"] else None)
    return state


# ---------------------------------------------------------------------------------------------- plain forms

def _keep(state, p):
    """The elements that dropout keeps, and what they are multiplied by: Philox4x32 of ten rounds, 16 bits per element."""
    case = state["case"]
    groups = (case["cols"] + 7) // 8
    n = torch.arange(case["rows"] * groups, device="cuda")
    low = 0xFFFFFFFF
    c0, c1 = n & low, n >> 32
    c2, c3 = torch.full_like(n, state["offset"] & low), torch.full_like(n, state["offset"] >> 32)
    k0, k1 = state["seed"] & low, state["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # 64-bit products; the shifts below take their bits as unsigned
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(case["rows"], 8 * groups)[:, : case["cols"]]
    least = round(p * 65536)
    return halves >= least, 65536 / (65536 - least)


def _drop(state, x, p):
    if p == 0:
        return x
    keep, factor = _keep(state, p)
    return torch.where(keep, x * factor, 0.0)


def _logits(state):
    return state["hidden"].float() @ state["weight"].float().T


def _plain_loss(state):
    case, targets = state["case"], state["targets"]
    z = _logits(state)
    most = z.max(1, keepdim=True).values
    lse = (most + (z - most).exp().sum(1, keepdim=True).log())[:, 0]
    valid = targets != IGNORE
    of_target = z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    loss = lse - (1 - case["smooth"]) * of_target + case["z"] * lse * lse
    if case["smooth"]:
        loss = loss - case["smooth"] * z.mean(1)
    return {"loss": torch.where(valid, loss, 0.0), "lse": torch.where(valid, lse, 0.0)}


def _plain_loss_grad(state):
    case, targets, lse = state["case"], state["targets"], state["lse"]
    d = (_logits(state) - lse[:, None]).exp_()
    if case["z"]:
        d *= (1 + 2 * case["z"] * lse)[:, None]
    if case["smooth"]:
        d -= case["smooth"] / case["vocab"]
    valid = targets != IGNORE
    d.scatter_add_(1, targets.clamp(min=0)[:, None], torch.full_like(lse, case["smooth"] - 1)[:, None])
    weight = valid * state["scale"]
    d *= (weight if state["dloss"] is None else weight * state["dloss"])[:, None]
    return {"dhidden": (d @ state["weight"].float()).to(TYPES[case["dhidden"]]),
            "dweight": (d.T @ state["hidden"].float()).to(TYPES[case["dweight"]])}


def _plain_norm(state):
    case = state["case"]
    kind = TYPES[case["type"]]
    s = _drop(state, state["x"].float(), case["p"])
    if state["residual"] is not None:
        s = s + state["residual"].float()
    rstd = (s.square().mean(1, keepdim=True) + case["eps"]).rsqrt()
    y = s * rstd * state["weight"].float()
    out = {"rstd": rstd[:, 0]}
    if state["residual"] is not None or case["p"]:
        out["sum"] = s.to(kind)
    if case["q8"] is None:
        out["y"] = y.to(kind)
        return out
    group = case["q8"] or case["cols"]
    n = -(-case["cols"] // group)
    y = torch.nn.functional.pad(y, (0, n * group - case["cols"])).view(case["rows"], n, group)
    most = y.abs().amax(2, keepdim=True)
    out["scale"] = torch.where(most > 0, most / 448, 1.0)[:, :, 0]
    q = (y * torch.where(most > 0, 448 / most, 1.0)).reshape(case["rows"], n * group)
    out["y8"] = q[:, : case["cols"]].contiguous().to(E4M3)
    return out


def _plain_norm_grad(state):
    case = state["case"]
    kind = TYPES[case["type"]]
    dy, xhat = state["dy"].float(), state["sum"].float() * state["rstd"][:, None]
    dyw = dy * state["weight"].float()
    ds = (dyw - xhat * (dyw * xhat).mean(1, keepdim=True)) * state["rstd"][:, None]
    if state["dsum"] is not None:
        ds = ds + state["dsum"].float()
    out = {"dresidual": ds.to(kind), "dweight": (dy * xhat).sum(0, dtype=torch.float64).to(TYPES[case["dweight"]])}
    if case["p"]:
        out["dx"] = _drop(state, ds, case["p"]).to(kind)
    return out


def _plain_dropout(state):
    y = _drop(state, state["x"].float(), state["case"]["p"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return {"y": y.to(TYPES[state["case"]["type"]])}


# ---------------------------------------------------------------------------------------------- the library's calls

def _own_loss_desc(A, state):
    """The descriptor, scratch and outputs that a program keeps from one call to the next."""
    kept, case = state["kept"], state["case"]
    if not kept:
        grad = case["op"] == "loss_grad"
        kept["desc"] = A.head_loss_desc(
            case["tokens"], case["vocab"], case["width"], hidden_ld=case["width"] + case["pad"], ignore_index=IGNORE,
            label_smoothing=case["smooth"], z_loss=case["z"],
            dhidden_dtype=A.TYPE_F32 if grad and case["dhidden"] == "f32" else A.TYPE_BF16,
            dweight_dtype=A.TYPE_F32 if grad and case["dweight"] == "f32" else A.TYPE_BF16)
        kept["scratch"] = torch.empty(A.adapm_head_loss_scratch_bytes(kept["desc"], grad), dtype=torch.uint8, device="cuda")
        if grad:
            kept["dhidden"] = torch.empty_strided((case["tokens"], case["width"]), (case["width"] + case["pad"], 1), dtype=TYPES[case["dhidden"]], device="cuda")
            kept["dweight"] = torch.empty(case["vocab"], case["width"], dtype=TYPES[case["dweight"]], device="cuda")
        else:
            kept["loss"], kept["lse"] = torch.empty(2, case["tokens"], device="cuda")
    return kept


def _own_loss(state):
    import paper_2510_09103_b200 as A
    k = _own_loss_desc(A, state)
    A.adapm_head_loss_forward(k["desc"], state["hidden"], state["weight"], state["targets"], k["loss"], k["lse"], k["scratch"])
    return {"loss": k["loss"], "lse": k["lse"]}


def _own_loss_grad(state):
    import paper_2510_09103_b200 as A
    k = _own_loss_desc(A, state)
    A.adapm_head_loss_backward(k["desc"], state["hidden"], state["weight"], state["targets"], state["lse"], state["dloss"],
                               state["scale"], k["dhidden"], k["dweight"], k["scratch"])
    return {"dhidden": k["dhidden"], "dweight": k["dweight"]}


def _own_norm_desc(A, state):
    kept, case = state["kept"], state["case"]
    if not kept:
        kept["desc"] = A.rmsnorm_desc(
            case["rows"], case["cols"], dtype=A.TYPE_F32 if case["type"] == "f32" else A.TYPE_BF16,
            weight_dtype=A.TYPE_F32 if case["weight"] == "f32" else A.TYPE_BF16, eps=case["eps"], drop_p=case["p"],
            seed=state["seed"], offset=state["offset"], q8_group=case.get("q8") or 0)
    return kept


def _own_norm(state):
    import paper_2510_09103_b200 as A
    case, k = state["case"], _own_norm_desc(A, state)
    if "rstd" not in k:
        new = lambda kind: torch.empty(case["rows"], case["cols"], dtype=kind, device="cuda")  # noqa: E731
        k["rstd"] = torch.empty(case["rows"], device="cuda")
        if state["residual"] is not None or case["p"]:
            k["sum"] = new(TYPES[case["type"]])
        if case["q8"] is None:
            k["y"] = new(TYPES[case["type"]])
        else:
            k["y8"] = new(E4M3)
            k["scale"] = torch.empty(case["rows"], -(-case["cols"] // (case["q8"] or case["cols"])), device="cuda")
    A.adapm_rmsnorm_forward(k["desc"], state["x"], state["residual"], state["weight"], k.get("sum"), k.get("y"), k.get("y8"),
                            k.get("scale"), k["rstd"])
    return {name: k[name] for name in ("rstd", "sum", "y", "y8", "scale") if name in k}


def _own_norm_grad(state):
    import paper_2510_09103_b200 as A
    case, k = state["case"], _own_norm_desc(A, state)
    if "dweight" not in k:
        k["dresidual"] = torch.empty_like(state["sum"])
        if case["p"]:
            k["dx"] = torch.empty_like(state["sum"])
        k["dweight"] = torch.empty(case["cols"], dtype=TYPES[case["dweight"]], device="cuda")
        k["scratch"] = torch.empty(A.adapm_rmsnorm_backward_scratch_bytes(k["desc"]), dtype=torch.uint8, device="cuda")
    A.adapm_rmsnorm_backward(k["desc"], state["dy"], state["dsum"], state["sum"], state["rstd"], state["weight"], k["dresidual"],
                             k.get("dx"), k["dweight"], A.TYPE_F32 if case["dweight"] == "f32" else A.TYPE_BF16, False, k["scratch"])
    return {name: k[name] for name in ("dresidual", "dweight", "dx") if name in k}


def _own_dropout(state):
    import paper_2510_09103_b200 as A
    case, k = state["case"], state["kept"]
    if not k:
        k["y"] = torch.empty_like(state["x"])
    A.adapm_dropout(state["x"], state["residual"], k["y"], A.TYPE_F32 if case["type"] == "f32" else A.TYPE_BF16, case["rows"],
                    case["cols"], case["p"], state["seed"], state["offset"])
    return {"y": k["y"]}


PLAIN = {"loss": _plain_loss, "loss_grad": _plain_loss_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "dropout": _plain_dropout}
OWN = {"loss": _own_loss, "loss_grad": _own_loss_grad, "norm": _own_norm, "norm_grad": _own_norm_grad, "dropout": _own_dropout}


def run(state):
    op = state["case"]["op"]
    return OWN[op](state) if own else PLAIN[op](state)


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] in ("loss", "loss_grad"):
        tokens, vocab, width = _valid(case), case["vocab"], case["width"]
        moved, flops = 2 * (tokens + vocab) * width + 8 * case["tokens"], 2.0 * tokens * vocab * width
        if case["op"] == "loss":
            return {"bytes": moved + 8 * case["tokens"], "flops": flops}
        moved += 4 * case["tokens"] * (2 if case["weighted"] else 1)
        moved += size[case["dhidden"]] * case["tokens"] * width + size[case["dweight"]] * vocab * width
        return {"bytes": moved, "flops": 3 * flops}
    elems, each = case["rows"] * case["cols"], size[case["type"]]
    if case["op"] == "dropout":
        return {"bytes": elems * each * (3 if case["residual"] else 2), "flops": 0}
    moved = size[case["weight"]] * case["cols"] + 4 * case["rows"]
    if case["op"] == "norm":
        moved += elems * each * (1 + case["residual"] + (case["residual"] or case["p"] > 0))
        if case["q8"] is None:
            return {"bytes": moved + elems * each, "flops": 0}
        groups = -(-case["cols"] // (case["q8"] or case["cols"]))
        return {"bytes": moved + elems + 4 * case["rows"] * groups, "flops": 0}
    moved += size[case["dweight"]] * case["cols"]
    return {"bytes": moved + elems * each * (3 + case["residual"] + (case["p"] > 0)), "flops": 0}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits

def _times_high(a, m):
    """Upper 32 bits of the product of 32-bit numbers, by parts of 16 bits."""
    al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    middle = ah * ml + ((al * ml) >> 16)
    return ah * mh + (middle >> 16) + (((middle & 0xFFFF) + al * mh) >> 16)


def _exact_drop(state, x):
    case = state["case"]
    if not case["p"]:
        return x
    col = torch.arange(case["cols"], device="cuda")
    row = torch.arange(case["rows"], device="cuda")
    # one counter per group of eight columns, in a table [rows, groups]; element (row, col) then looks its 16 bits up
    ctr = row[:, None] * ((case["cols"] + 7) // 8) + torch.arange((case["cols"] + 7) // 8, device="cuda")
    key, mask = [state["seed"] % 2**32, state["seed"] // 2**32], 2**32 - 1
    words = [ctr % 2**32, ctr // 2**32, state["offset"] % 2**32 + 0 * ctr, state["offset"] // 2**32 + 0 * ctr]
    for r in range(10):
        k = [(key[0] + r * 0x9E3779B9) & mask, (key[1] + r * 0xBB67AE85) & mask]
        h0, l0 = _times_high(words[0], 0xD2511F53), (words[0] * 0xD2511F53) & mask
        h1, l1 = _times_high(words[2], 0xCD9E8D57), (words[2] * 0xCD9E8D57) & mask
        words = [h1 ^ words[1] ^ k[0], l1, h0 ^ words[3] ^ k[1], l0]
    bits = torch.empty(case["rows"], case["cols"], dtype=torch.int64, device="cuda")
    for j in range(8):
        at = col[col % 8 == j]
        bits[:, at] = ((words[j // 2] >> (16 * (j % 2))) & 0xFFFF)[:, at // 8]
    least = round(case["p"] * 65536)
    return x.masked_fill(bits < least, 0.0) / (1 - least / 65536)


def exact(case, seed):
    state = prepare(case, seed)
    wide = {k: v.double() for k, v in state.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] in ("loss", "loss_grad"):
        valid = (state["targets"] != IGNORE).nonzero()[:, 0]
        outs = {}
        if case["op"] == "loss_grad":
            outs = {"dhidden": torch.zeros_like(wide["hidden"]), "dweight": torch.zeros_like(wide["weight"])}
        else:
            outs = {"loss": torch.zeros(case["tokens"], dtype=torch.float64, device="cuda"), "lse": torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")}
        for at in valid.split(1024):
            h, y = wide["hidden"][at], state["targets"][at]
            z = torch.einsum("td,vd->tv", h, wide["weight"])
            if case["op"] == "loss":
                lse = torch.logsumexp(z, 1)
                aim = torch.full_like(z, case["smooth"] / case["vocab"])
                aim[torch.arange(len(at), device="cuda"), y] += 1 - case["smooth"]
                outs["lse"][at], outs["loss"][at] = lse, -(aim * (z - lse[:, None])).sum(1) + case["z"] * lse**2
                continue
            lse = wide["lse"][at]
            g = torch.exp(z - lse[:, None]) * (1 + 2 * case["z"] * lse)[:, None] - case["smooth"] / case["vocab"]
            g[torch.arange(len(at), device="cuda"), y] -= 1 - case["smooth"]
            g *= state["scale"]
            if state["dloss"] is not None:
                g *= wide["dloss"][at][:, None]
            outs["dhidden"][at] = torch.einsum("tv,vd->td", g, wide["weight"])
            outs["dweight"] += torch.einsum("tv,td->vd", g, h)
        return outs
    if case["op"] == "dropout":
        y = _exact_drop(state, wide["x"])
        return {"y": y if state["residual"] is None else y + wide["residual"]}
    if case["op"] == "norm":
        s = _exact_drop(state, wide["x"])
        s = s if state["residual"] is None else s + wide["residual"]
        rms = torch.sqrt(torch.linalg.vector_norm(s, dim=1) ** 2 / case["cols"] + case["eps"])
        y = s / rms[:, None] * wide["weight"]
        out = {"rstd": 1 / rms}
        if state["residual"] is not None or case["p"]:
            out["sum"] = s
        if case["q8"] is None:
            return dict(out, y=y)
        scales = [part.abs().amax(1) / 448 for part in y.split(case["q8"] or case["cols"], 1)]
        scale = torch.stack([torch.where(m == 0, 1.0, m) for m in scales], 1)
        return dict(out, scale=scale, y8=y / scale.repeat_interleave(case["q8"] or case["cols"], 1)[:, : case["cols"]])
    # the gradient of sum(dy * y) + sum(dsum * s) with respect to s, from y_i = w_i s_i rstd and d rstd / d s_j = -rstd^3 s_j / cols
    dy, s, rstd, w = wide["dy"], wide["sum"], wide["rstd"][:, None], wide["weight"]
    inner = torch.einsum("rc,rc,c->r", dy, s, w)[:, None]
    ds = dy * w * rstd - s * rstd**3 * inner / case["cols"]
    if state["dsum"] is not None:
        ds = ds + wide["dsum"]
    out = {"dresidual": ds, "dweight": torch.einsum("rc,rc,ro->c", dy, s, rstd)}
    if case["p"]:
        out["dx"] = _exact_drop(state, ds)
    return out
