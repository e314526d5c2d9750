"""The operators for models that train on decoded images as packed patch tokens, as cases that can
be timed and compared: patch tokens, dropout, rotary positions, norms of queries and keys with the
rotation, attention over packed images (forward, with its gradients, and for single tokens).

`own` chooses what `run` does: the plain form, elementary torch operations in 32 bits (angles in 64),
or the library's calls.  `exact` works the same outputs out in 64 bits, written apart from both.
"""
import math
import random

import torch

own = False

MEAN, STDV = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- the cases --------------------------------------------------------------------------------


def _tokens(name, images, width, height, side, dtype):
    """width and height are ranges: (least, most) of the images of a batch."""
    return {"name": name, "op": "tokens", "images": images, "width_min": width[0], "width_max": width[1],
            "height_min": height[0], "height_max": height[1], "side": side, "dtype": dtype}


def _dropout(name, rows, cols, dtype, p, residual):
    return {"name": name, "op": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _rotate(name, tokens, heads, head_dim, pairs, dtype, **more):
    """norm: queries and keys are normalised first; back: the gradients' way.  axes 2: row and column
    of an image's patches; axes 1: one position, up to `last`.  factor > 1: trained on `original`
    positions and stretched by it."""
    case = {"name": name, "op": "rotate", "tokens": tokens, "q_heads": heads[0], "k_heads": heads[1], "head_dim": head_dim,
            "pairs": pairs, "dtype": dtype, "norm": False, "back": False, "axes": 2, "interleaved": False,
            "last": 1, "factor": 1.0, "original": 0}
    case.update(more)
    return case


def _attention(name, images, length, heads, head_dim, dtype, **more):
    """length: range of an image's tokens.  train: the gradients too.  mask: what a token sees of
    its own image: all of it ("document"), what comes before it ("causal"), or that and a prefix
    that all see ("prefix")."""
    case = {"name": name, "op": "attention", "images": images, "length_min": length[0], "length_max": length[1],
            "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "dtype": dtype, "train": False,
            "mask": "document", "cap": 0.0, "slopes": False}
    case.update(more)
    return case


def _step(name, images, length, heads, head_dim, dtype, **more):
    """One token a sequence against caches whose lengths lie in `length`."""
    case = _attention(name, images, length, heads, head_dim, dtype, op="step", mask="causal")
    del case["train"]
    case.update(more)
    return case


def listed():
    return [
        # a small per-GPU share of street scenes, cut into 16x16 patches for an encoder
        _tokens("tokens_street_4", 4, (2048, 2048), (1024, 1024), 16, "bf16"),
        # a classification batch of photographs of all sizes; patches of 14, ragged at the edges
        _tokens("tokens_photos_256", 256, (400, 500), (300, 375), 14, "fp16"),
        # one photograph's tokens behind the embedding: what a call costs
        _dropout("dropout_one_photo", 616, 768, "bf16", 0.1, False),
        # a training batch behind a block, added to the residual stream
        _dropout("dropout_batch", 65536, 1024, "fp16", 0.25, True),
        # the gradient's way of a 64x64 image's patches (16 tokens): what a call costs
        _rotate("rotate_small_back", 16, (12, 12), 64, 32, "fp16", back=True),
        # far positions of a long context, part of the head, pairs side by side, stretched eight times
        _rotate("rotate_long", 65536, (32, 8), 128, 32, "bf16", axes=1, interleaved=True, last=1 << 20, factor=8.0,
                original=8192),
        # queries and keys of a training batch straight out of the joint projection
        _rotate("norm_rotate_batch", 40000, (12, 12), 64, 32, "bf16", norm=True),
        # their gradients and the norms' weights', with fewer heads of keys; odd number of tokens
        _rotate("norm_rotate_back", 19683, (16, 2), 128, 64, "bf16", norm=True, back=True),
        # one small, one odd and one single-token image with a head that is no power of two: latency
        _attention("attention_small", 3, (1, 197), (6, 6), 72, "fp16", mask="prefix", cap=30.0),
        # a batch of photographs of all sizes packed end to end, forward
        _attention("attention_photos_64", 64, (400, 768), (12, 12), 64, "bf16"),
        # street scenes of 8192 patches each, forward and gradients, shared heads, causal and capped
        _attention("attention_street_train", 4, (7000, 8192), (16, 2), 128, "bf16", train=True, mask="causal", cap=50.0),
        # one more token for each of 32 sequences with caches of all lengths, biased by distance
        _step("step_32", 32, (512, 32768), (32, 8), 128, "bf16", slopes=True),
    ]


def _log_uniform(rng, least, most):
    return max(least, min(most, int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))))


def draw(rng):
    op = rng.choice(("tokens", "dropout", "rotate", "norm_rotate", "attention", "attention", "train", "train", "step", "step"))
    dtype = rng.choice(("bf16", "fp16"))
    if op == "tokens":
        width = _log_uniform(rng, 40, 2048)
        height = max(24, min(1024, int(width * rng.uniform(0.45, 1.3))))
        low = rng.choice((1.0, 0.7))
        images = max(1, min(256, _log_uniform(rng, width * height, 30_000_000) // (width * height)))
        case = _tokens("", images, (int(width * low), width), (int(height * low), height), rng.choice((8, 14, 16, 16, 28, 7)), dtype)
    elif op == "dropout":
        cols = rng.choice((64, 192, 384, 513, 768, 1000, 1024, 2048, 4096))
        rows = max(1, _log_uniform(rng, 500, 60_000_000) // cols)
        case = _dropout("", rows, cols, dtype, rng.choice((0.05, 0.1, 0.25, 0.5, 0.9)), rng.random() < 0.5)
    elif op in ("rotate", "norm_rotate"):
        head_dim = rng.choice((32, 64, 64, 72, 80, 88, 128, 128))
        kv = rng.choice((1, 2, 4, 8, 12))
        heads = (kv * rng.choice((1, 1, 2, 4)), kv)
        tokens = max(1, _log_uniform(rng, 1, 60_000_000 // ((heads[0] + heads[1]) * head_dim)))
        axes = rng.choice((1, 2))
        pairs = rng.choice((head_dim // 2, head_dim // 4))
        stretched = axes == 1 and rng.random() < 0.5
        case = _rotate("", tokens, heads, head_dim, pairs // axes * axes, dtype, norm=op == "norm_rotate",
                       back=rng.random() < 0.5, axes=axes, interleaved=rng.random() < 0.5,
                       last=_log_uniform(rng, tokens, 1 << 20) if axes == 1 else 1,
                       factor=float(rng.choice((2, 4, 8))) if stretched else 1.0, original=8192 if stretched else 0)
    elif op == "step":
        kv = rng.choice((1, 2, 4, 8))
        heads = (kv * rng.choice((1, 2, 4, 8)), kv)
        head_dim = rng.choice((64, 64, 80, 128, 128))
        images = _log_uniform(rng, 1, 64)
        most = _log_uniform(rng, 1, min(131072, 300_000_000 // (images * kv * head_dim)))
        case = _step("", images, (max(1, int(most * rng.choice((0.05, 0.5, 1.0)))), most), heads, head_dim, dtype,
                     cap=rng.choice((0.0, 30.0)), slopes=rng.random() < 0.5)
    else:
        kv = rng.choice((1, 2, 3, 4, 8))
        heads = (kv * rng.choice((1, 1, 2, 4)), kv)
        head_dim = rng.choice((32, 64, 64, 72, 80, 128, 128))
        most = _log_uniform(rng, 1, 6000)
        # products of queries and keys, at most half of the largest listed case's
        images = max(1, min(300, int(_log_uniform(rng, 1000, 1_000_000_000) * 8 / heads[0] / (most * most)), 1))
        images = min(max(images, _log_uniform(rng, 1, 64)), max(1, 60_000_000 // (most * heads[0] * head_dim)))
        images = max(1, min(images, int(2_000_000_000 / heads[0]) // (most * most)))
        case = _attention("", images, (max(1, int(most * rng.choice((0.1, 0.6, 1.0)))), most), heads, head_dim, dtype,
                          train=op == "train", mask=rng.choice(("document", "document", "causal", "prefix")),
                          cap=rng.choice((0.0, 0.0, 30.0)), slopes=rng.random() < 0.3)
    del case["name"]
    return case


# ---- inputs -----------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    return gen


def _sizes(case, key, low, high):
    """Sizes that belong to the case, not to the seed, so that outputs of two seeds have one shape."""
    rng = random.Random(case["images"] * 65537 + high * 31 + low + key)
    return [rng.randint(low, high) for _ in range(case["images"])]


def _image_shapes(case):
    return list(zip(_sizes(case, 1, case["width_min"], case["width_max"]), _sizes(case, 2, case["height_min"], case["height_max"])))


def _lengths(case):
    lengths = _sizes(case, 3, case["length_min"], case["length_max"])
    lengths[0] = case["length_max"]
    if case["images"] >= 3 and case["length_min"] == 1:
        lengths[1] = 1
    return lengths


def _first(lengths):
    """Where each sequence starts, and the end of the last."""
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _frequencies(case):
    """Radians a position, one per pair of an axis.  Stretched contexts: a pair that turns often
    over the original context keeps its frequency, one that hardly turns is slowed down by the
    factor, with a ramp between 32 turns and 1."""
    m = case["pairs"] // case["axes"]
    out = []
    for j in range(m):
        f = 10000.0 ** (-j / m)
        if case["factor"] > 1.0:
            turns = case["original"] * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            f = f * (keep + (1.0 - keep) / case["factor"])
        out.append(f)
    return out * case["axes"]


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0


def _slopes(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


_contexts = {}


def _context():
    """One context a process, as a user's program keeps it."""
    import paper_2208_08711_amd as l3
    device = torch.cuda.current_device()
    if device not in _contexts:
        _contexts[device] = l3.Context(device)
    return _contexts[device]


def _normal(shape, gen, dtype):
    """Normal values of the type, made in pieces so that no large 32-bit copy stands beside them."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        piece = flat[at:at + (1 << 26)]
        piece.copy_(torch.randn(piece.numel(), generator=gen, device="cuda"))
    return out


def prepare(case, seed):
    gen = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    state = {"case": case, "seed": seed}
    if own:
        state["context"] = _context()
    if case["op"] == "tokens":
        shapes = _image_shapes(case)
        flat = torch.randint(0, 256, (sum(3 * w * h for w, h in shapes),), generator=gen, device="cuda", dtype=torch.uint8)
        images, at = [], 0
        for w, h in shapes:
            images.append(flat[at:at + 3 * w * h].view(h, w, 3))
            at += 3 * w * h
        state["images"] = images
        side = case["side"]
        total = sum(-(-w // side) * -(-h // side) for w, h in shapes)
        state["tokens"] = torch.empty((total, 3 * side * side), dtype=dtype, device="cuda")
        state["positions"] = torch.empty((total, 2), dtype=torch.int32, device="cuda")
        state["first"] = torch.empty(len(shapes) + 1, dtype=torch.int32, device="cuda")
    elif case["op"] == "dropout":
        shape = (case["rows"], case["cols"])
        state["x"] = _normal(shape, gen, dtype)
        state["residual"] = _normal(shape, gen, dtype) if case["residual"] else None
        state["key"], state["offset"] = 0x9E3779B97F4A7C15 ^ seed, 3 * seed + 1
        state["out"] = torch.empty_like(state["x"])
    elif case["op"] == "rotate":
        t, hq, hk, d = case["tokens"], case["q_heads"], case["k_heads"], case["head_dim"]
        joint = _normal((t, hq + 2 * hk, d), gen, dtype)                 # queries, keys, values of the projection
        state["q"], state["k"] = joint[:, :hq], joint[:, hq:hq + hk]
        if case["axes"] == 2:                                            # patches of images about 32 across
            across = 32 + seed % 3
            at = torch.arange(t, device="cuda") % (across * across)
            state["positions"] = torch.stack((at // across, at % across), 1).to(torch.int32)
        else:
            start = max(0, case["last"] - t) - seed % 5
            state["positions"] = (torch.arange(t, device="cuda") + max(0, start)).to(torch.int32)
        if case["norm"]:
            state["q_weight"] = 1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")
            state["k_weight"] = 1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")
            if case["back"]:
                state["q_grad"], state["k_grad"] = _normal((t, hq, d), gen, dtype), _normal((t, hk, d), gen, dtype)
        state["q_out"] = torch.empty((t, hq, d), dtype=dtype, device="cuda")
        state["k_out"] = torch.empty((t, hk, d), dtype=dtype, device="cuda")
        if own:
            import paper_2208_08711_amd as l3
            m = case["pairs"] // case["axes"]
            table = l3.rotation_turns(m, 10000.0, factor=case["factor"], original_length=case["original"])
            state["rotation"] = l3.Rotation(list(table) * case["axes"], axes=case["axes"], interleaved=case["interleaved"],
                                            magnitude=_magnitude(case))
    elif case["op"] == "attention":
        lengths = _lengths(case)
        t, hq, hk, d = sum(lengths), case["q_heads"], case["kv_heads"], case["head_dim"]
        joint = _normal((t, hq + 2 * hk, d), gen, dtype)
        state["q"], state["k"], state["v"] = joint[:, :hq], joint[:, hq:hq + hk], joint[:, hq + hk:]
        state["host_first"] = _first(lengths)
        state["first"] = torch.tensor(state["host_first"], dtype=torch.int32, device="cuda")
        state["host_prefix"] = [(n * 2 + 4) // 5 for n in lengths] if case["mask"] == "prefix" else None
        state["prefix"] = torch.tensor(state["host_prefix"], dtype=torch.int32, device="cuda") if case["mask"] == "prefix" else None
        state["slopes"] = torch.tensor(_slopes(hq), device="cuda") if case["slopes"] else None
        state["out"] = torch.empty((t, hq, d), dtype=dtype, device="cuda")
        if case["train"]:
            state["grad"] = _normal((t, hq, d), gen, dtype)
            state["lse"] = torch.empty((hq, t), device="cuda")
            joint_grad = torch.empty_like(joint)
            state["q_grad"], state["k_grad"], state["v_grad"] = joint_grad[:, :hq], joint_grad[:, hq:hq + hk], joint_grad[:, hq + hk:]
    else:
        lengths = _lengths(case)
        n, hq, hk, d, room = case["images"], case["q_heads"], case["kv_heads"], case["head_dim"], case["length_max"]
        state["q"] = _normal((n, hq, d), gen, dtype)
        state["k"], state["v"] = _normal((n, room, hk, d), gen, dtype), _normal((n, room, hk, d), gen, dtype)
        state["host_lengths"] = lengths
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        state["slopes"] = torch.tensor(_slopes(hq), device="cuda") if case["slopes"] else None
        state["out"] = torch.empty((n, hq, d), dtype=dtype, device="cuda")
    return state


# ---- one pass ---------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return {"tokens": _own_tokens, "dropout": _own_dropout, "rotate": _own_rotate, "attention": _own_attention,
                "step": _own_step}[op](state)
    return {"tokens": _plain_tokens, "dropout": _plain_dropout, "rotate": _plain_rotate, "attention": _plain_attention,
            "step": _plain_step}[op](state)


def _own_tokens(state):
    import paper_2208_08711_amd as l3
    l3.patch_tokens_batch(state["context"], state["images"], state["case"]["side"], MEAN, STDV, state["tokens"],
                          positions=state["positions"], first=state["first"])
    return {"tokens": state["tokens"], "positions": state["positions"], "first": state["first"]}


def _own_dropout(state):
    import paper_2208_08711_amd as l3
    l3.dropout(state["context"], state["x"], state["out"], state["case"]["p"], state["key"], offset=state["offset"],
               residual=state["residual"])
    return state["out"]


def _own_rotate(state):
    import paper_2208_08711_amd as l3
    case = state["case"]
    outs = {"q": state["q_out"], "k": state["k_out"]}
    if not case["norm"]:
        l3.rotate(state["context"], state["rotation"], state["positions"], state["q"], state["q_out"], state["k"], state["k_out"],
                  inverse=case["back"])
    elif not case["back"]:
        l3.norm_rotate(state["context"], state["rotation"], state["positions"], state["q"], state["q_weight"], state["q_out"],
                       state["k"], state["k_weight"], state["k_out"], eps=EPS)
    else:
        outs["q_weight"] = torch.empty_like(state["q_weight"])
        outs["k_weight"] = torch.empty_like(state["k_weight"])
        l3.norm_rotate_backward(state["context"], state["rotation"], state["positions"],
                                state["q"], state["q_weight"], state["q_grad"], state["q_out"], outs["q_weight"],
                                state["k"], state["k_weight"], state["k_grad"], state["k_out"], outs["k_weight"], eps=EPS)
    return outs


def _own_attention(state):
    import paper_2208_08711_amd as l3
    case = state["case"]
    how = {"mask": {"document": l3.MASK_DOCUMENT, "causal": l3.MASK_CAUSAL, "prefix": l3.MASK_PREFIX}[case["mask"]],
           "prefix": state["prefix"], "cap": case["cap"], "slopes": state["slopes"]}
    if not case["train"]:
        l3.attention(state["context"], state["q"], state["k"], state["v"], state["out"], state["first"], **how)
        return {"out": state["out"]}
    l3.attention(state["context"], state["q"], state["k"], state["v"], state["out"], state["first"], lse=state["lse"], **how)
    l3.attention_backward(state["context"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["grad"],
                          state["q_grad"], state["k_grad"], state["v_grad"], state["first"], **how)
    return {"out": state["out"], "q_grad": state["q_grad"], "k_grad": state["k_grad"], "v_grad": state["v_grad"]}


def _own_step(state):
    import paper_2208_08711_amd as l3
    l3.attention_step(state["context"], state["q"], state["k"], state["v"], state["lengths"], state["out"],
                      cap=state["case"]["cap"], slopes=state["slopes"])
    return {"out": state["out"]}


def _plain_tokens(state):
    case, side = state["case"], state["case"]["side"]
    dtype = DTYPES[case["dtype"]]
    mean = torch.tensor(MEAN, device="cuda")
    stdv = torch.tensor(STDV, device="cuda")
    tokens, positions, first = [], [], [0]
    for image in state["images"]:
        h, w = image.shape[:2]
        rows, cols = -(-h // side), -(-w // side)
        padded = torch.zeros((rows * side, cols * side, 3), device="cuda")
        padded[:h, :w] = (image.float() / 255.0 - mean) / stdv
        cut = padded.view(rows, side, cols, side, 3).permute(0, 2, 4, 1, 3)
        tokens.append(cut.reshape(rows * cols, 3 * side * side).to(dtype))
        at = torch.arange(rows * cols, device="cuda", dtype=torch.int32)
        positions.append(torch.stack((at // cols, at % cols), 1))
        first.append(first[-1] + rows * cols)
    return {"tokens": torch.cat(tokens), "positions": torch.cat(positions),
            "first": torch.tensor(first, dtype=torch.int32).to("cuda", non_blocking=True)}


def _philox(blocks, key, offset):
    """Philox 4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3;
    SC 2011).  blocks: int64 tensor of the counter's low 64 bits.  Returns four int64 tensors below 2^32."""
    mask = 0xFFFFFFFF

    def product(a, b):
        """High and low 32 bits of a constant times a tensor below 2^32."""
        low = b * (a & 0xFFFF)
        high = b * (a >> 16)
        middle = (low >> 16) + (high & 0xFFFF)
        return (high >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (low & 0xFFFF)

    c0, c1 = blocks & mask, (blocks >> 32) & mask
    c2, c3 = torch.full_like(c0, offset & mask), torch.full_like(c0, (offset >> 32) & mask)
    k0, k1 = key & mask, (key >> 32) & mask
    for _ in range(7):
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c0, c1, c2, c3


def _kept(count, p, key, offset):
    """Truth value per element: element e has 16 bits of block e // 8, and stays if they reach p * 65536."""
    blocks = torch.arange((count + 7) // 8, device="cuda")
    words = torch.stack(_philox(blocks, key, offset), 1)
    halves = torch.stack((words & 0xFFFF, words >> 16), 2).view(-1)[:count]
    return halves >= int(p * 65536 + 0.5)


def _plain_dropout(state):
    x, p = state["x"], state["case"]["p"]
    kept = _kept(x.numel(), p, state["key"], state["offset"]).view(x.shape)
    scale = 65536.0 / (65536 - int(p * 65536 + 0.5))
    y = torch.where(kept, x.float() * scale, 0.0)
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return y.to(x.dtype)


def _angles(case, positions):
    """Cosines and sines [tokens, 1, pairs] in 32 bits, from angles in 64."""
    m = case["pairs"] // case["axes"]
    freq = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    p = positions.double().view(-1, case["axes"]).repeat_interleave(m, 1)
    angle = (p * freq)[:, None]
    return angle.cos().float(), angle.sin().float()


def _turned(x, cos, sin, case, back):
    """The rotation of the first 2 * pairs elements of every head, in 32 bits."""
    r = 2 * case["pairs"]
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
    if back:
        sin = -sin
    scale = _magnitude(case)
    c, d = (a * cos - b * sin) * scale, (a * sin + b * cos) * scale
    joined = torch.stack((c, d), -1).flatten(-2) if case["interleaved"] else torch.cat((c, d), -1)
    return torch.cat((joined, x[..., r:]), -1)


def _plain_rotate(state):
    case = state["case"]
    cos, sin = _angles(case, state["positions"])
    outs = {}
    for name in ("q", "k"):
        x = state[name].float()
        dtype = state[name].dtype
        if case["norm"]:
            weight = state[name + "_weight"]
            rstd = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
            if case["back"]:
                g = _turned(state[name + "_grad"].float(), cos, sin, case, True)
                n = x * rstd
                outs[name + "_weight"] = (g * n).sum((0, 1))
                g = g * weight
                x = rstd * (g - n * (g * n).mean(-1, keepdim=True))
            else:
                x = _turned(x * rstd * weight, cos, sin, case, False)
        else:
            x = _turned(x, cos, sin, case, case["back"])
        outs[name] = x.to(dtype)
    return outs


def _visible(case, state, image, queries, keys):
    """What the queries of an image see, [queries, keys], or None for all of it."""
    if case["mask"] == "document":
        return None
    i = torch.arange(queries, device="cuda")[:, None]
    j = torch.arange(keys, device="cuda")
    seen = j <= i
    if case["mask"] == "prefix":
        seen = seen | (j < state["host_prefix"][image])
    return seen


def _plain_attention(state):
    case = state["case"]
    q, k, v = state["q"], state["k"], state["v"]
    dtype, d = q.dtype, case["head_dim"]
    group, scale, cap = case["q_heads"] // case["kv_heads"], 1.0 / math.sqrt(d), case["cap"]
    outs = {"out": torch.empty(q.shape, dtype=dtype, device="cuda")}
    if case["train"]:
        for name, x in (("q_grad", q), ("k_grad", k), ("v_grad", v)):
            outs[name] = torch.empty(x.shape, dtype=dtype, device="cuda")
    first = state["host_first"]
    for image in range(case["images"]):
        rows = slice(first[image], first[image + 1])
        n = first[image + 1] - first[image]
        if n == 0:
            continue
        seen = _visible(case, state, image, n, n)
        far = None
        if state["slopes"] is not None:
            at = torch.arange(n, device="cuda")
            far = (at[:, None] - at).abs().float()
        for kv in range(case["kv_heads"]):
            heads = slice(kv * group, (kv + 1) * group)
            qh = q[rows, heads].float().transpose(0, 1).contiguous()             # [group, n, d]
            kh, vh = k[rows, kv].float().contiguous(), v[rows, kv].float().contiguous()
            raw = torch.matmul(qh, kh.t().contiguous()) * scale
            s = torch.tanh(raw / cap) * cap if cap else raw
            slope = (1.0 - (s / cap).square()) if cap and case["train"] else None
            del raw
            if far is not None:
                s = s - state["slopes"][heads, None, None] * far
            if seen is not None:
                s = s.masked_fill(~seen, float("-inf"))
            s = s - s.amax(-1, keepdim=True)
            w = s.exp()
            w = w / w.sum(-1, keepdim=True)
            out = torch.matmul(w, vh)
            outs["out"][rows, heads] = out.transpose(0, 1).to(dtype)
            if case["train"]:
                g = state["grad"][rows, heads].float().transpose(0, 1).contiguous()
                outs["v_grad"][rows, kv] = torch.matmul(w.transpose(1, 2).contiguous(), g).sum(0).to(dtype)
                ds = w * (torch.matmul(g, vh.t().contiguous()) - (g * out).sum(-1, keepdim=True))
                if slope is not None:
                    ds = ds * slope
                ds = ds * scale
                outs["q_grad"][rows, heads] = torch.matmul(ds, kh).transpose(0, 1).to(dtype)
                outs["k_grad"][rows, kv] = torch.matmul(ds.transpose(1, 2).contiguous(), qh).sum(0).to(dtype)
    return outs


def _plain_step(state):
    case = state["case"]
    q = state["q"]
    d, group = case["head_dim"], case["q_heads"] // case["kv_heads"]
    out = torch.empty_like(q)
    for image, n in enumerate(state["host_lengths"]):
        qh = q[image].float().view(case["kv_heads"], group, d)
        kh = state["k"][image, :n].float().permute(1, 2, 0).contiguous()         # [kv_heads, d, n]
        vh = state["v"][image, :n].float().transpose(0, 1).contiguous()
        s = torch.matmul(qh, kh) / math.sqrt(d)
        if case["cap"]:
            s = torch.tanh(s / case["cap"]) * case["cap"]
        if state["slopes"] is not None:
            far = (n - 1 - torch.arange(n, device="cuda")).float()
            s = s - state["slopes"].view(case["kv_heads"], group, 1) * far
        s = (s - s.amax(-1, keepdim=True)).exp()
        out[image] = (torch.matmul(s, vh) / s.sum(-1, keepdim=True)).view(-1, d).to(q.dtype)
    return {"out": out}


# ---- the same in 64 bits ----------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return {"tokens": _exact_tokens, "dropout": _exact_dropout, "rotate": _exact_rotate, "attention": _exact_attention,
            "step": _exact_step}[case["op"]](case, state)


def _exact_tokens(case, state):
    side = case["side"]
    table = [[(v / 255.0 - MEAN[c]) / STDV[c] for v in range(256)] for c in range(3)]
    table = torch.tensor(table, dtype=torch.float64, device="cuda")
    parts = []
    for image in state["images"]:
        h, w = image.shape[:2]
        planes = torch.stack([table[c][image[:, :, c].long()] for c in range(3)])
        planes = torch.nn.functional.pad(planes, (0, -w % side, 0, -h % side))
        cut = planes.unfold(1, side, side).unfold(2, side, side)                 # [3, rows, cols, side, side]
        parts.append(cut.permute(1, 2, 0, 3, 4).reshape(-1, 3 * side * side))
    return {"tokens": torch.cat(parts), "positions": None, "first": None}


def _exact_dropout(case, state):
    x = state["x"].double()
    # the generator once more, a 64-bit product at a time in two's complement
    count = x.numel()
    n = torch.arange((count + 7) // 8, device="cuda")
    word = 1 << 32
    c = [n % word, n // word, torch.full_like(n, state["offset"] % word), torch.full_like(n, state["offset"] // word)]
    k = [state["key"] % word, state["key"] // word]
    for r in range(7):
        lows, highs = [], []
        for m, v in ((0xD2511F53, c[0]), (0xCD9E8D57, c[2])):
            half = v * (m >> 1)                                                  # below 2^63
            low = (((half % word) * 2) + (v if m & 1 else 0))
            highs.append((half // word) * 2 + low // word)
            lows.append(low % word)
        c = [highs[1] ^ c[1] ^ ((k[0] + r * 0x9E3779B9) % word), lows[1], highs[0] ^ c[3] ^ ((k[1] + r * 0xBB67AE85) % word), lows[0]]
    bits = torch.empty((n.numel(), 8), dtype=torch.int64, device="cuda")
    for i in range(8):
        bits[:, i] = (c[i // 2] >> (16 * (i % 2))) % 65536
    t = int(case["p"] * 65536 + 0.5)
    y = x * (65536.0 / (65536 - t)) * (bits.view(-1)[:count].view(x.shape) >= t)
    return y if state["residual"] is None else y + state["residual"].double()


def _exact_rotate(case, state):
    """As complex numbers: a pair is a + ib, the rotation a product with exp(i angle)."""
    m, r = case["pairs"] // case["axes"], 2 * case["pairs"]
    freq = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    at = state["positions"].reshape(-1, case["axes"]).double()
    angle = torch.cat([at[:, a:a + 1] * freq[a * m:(a + 1) * m] for a in range(case["axes"])], 1)
    turn = torch.polar(torch.full_like(angle, _magnitude(case)), -angle if case["back"] else angle)[:, None]

    def rotated(x):
        x = x.clone()
        first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    outs = {}
    for name in ("q", "k"):
        x = state[name].double()
        if not case["norm"]:
            outs[name] = rotated(x)
            continue
        w = state[name + "_weight"].double()
        norm = torch.sqrt((x * x).sum(-1, keepdim=True) / case["head_dim"] + EPS)
        if not case["back"]:
            outs[name] = rotated(x / norm * w)
            continue
        g = rotated(state[name + "_grad"].double())
        outs[name + "_weight"] = (g * x / norm).sum((0, 1))
        dot = (g * w * x).sum(-1, keepdim=True)
        outs[name] = g * w / norm - x * dot / (case["head_dim"] * norm ** 3)
    return outs


def _exact_attention(case, state):
    d = case["head_dim"]
    group = case["q_heads"] // case["kv_heads"]
    first = state["host_first"]
    q, k, v = state["q"], state["k"], state["v"]
    shape = {"out": q.shape}
    if case["train"]:
        shape.update(q_grad=q.shape, k_grad=k.shape, v_grad=v.shape)
    outs = {name: torch.zeros(s, dtype=torch.float64, device="cuda") for name, s in shape.items()}
    for image in range(case["images"]):
        a, b = first[image], first[image + 1]
        n = b - a
        index = torch.arange(n, device="cuda")
        hidden = None
        if case["mask"] != "document":
            limit = index + 1
            if case["mask"] == "prefix":
                limit = limit.clamp(min=state["host_prefix"][image])
            hidden = index[None] >= limit[:, None]
        for h in range(case["q_heads"]):
            kv = h // group
            qh, kh, vh = q[a:b, h].double(), k[a:b, kv].double(), v[a:b, kv].double()
            s = torch.mm(qh, kh.t().contiguous()) * d ** -0.5
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
                steep = 1 - (s / case["cap"]) ** 2
            if state["slopes"] is not None:
                s = s - float(state["slopes"][h]) * (index[:, None] - index[None]).abs()
            if hidden is not None:
                s[hidden] = -math.inf
            p = torch.softmax(s, -1)
            del s
            out = torch.mm(p, vh)
            outs["out"][a:b, h] = out
            if not case["train"]:
                continue
            g = state["grad"][a:b, h].double()
            outs["v_grad"][a:b, kv] += torch.mm(p.t().contiguous(), g)
            p *= torch.mm(g, vh.t().contiguous()) - (g * out).sum(1, keepdim=True)
            if case["cap"]:
                p *= steep
            p *= d ** -0.5
            outs["q_grad"][a:b, h] = torch.mm(p, kh)
            outs["k_grad"][a:b, kv] += torch.mm(p.t().contiguous(), qh)
    return outs


def _exact_step(case, state):
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    for image, n in enumerate(state["host_lengths"]):
        for h in range(case["q_heads"]):
            k, v = state["k"][image, :n, h // group].double(), state["v"][image, :n, h // group].double()
            s = torch.mv(k, state["q"][image, h].double()) * case["head_dim"] ** -0.5
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            if state["slopes"] is not None:
                s = s + float(state["slopes"][h]) * (torch.arange(n, device="cuda") - (n - 1))
            out[image, h] = torch.softmax(s, 0) @ v
    return {"out": out}


# ---- what a pass cannot do without ------------------------------------------------------------


def work(case):
    if case["op"] == "tokens":
        side = case["side"]
        shapes = _image_shapes(case)
        pixels = sum(w * h for w, h in shapes)
        total = sum(-(-w // side) * -(-h // side) for w, h in shapes)
        return {"bytes": 3 * pixels + total * (6 * side * side + 8) + 4 * (len(shapes) + 1), "flops": 0}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (6 if case["residual"] else 4), "flops": (3 if case["residual"] else 2) * n}
    if case["op"] == "rotate":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        moved = 6 if case["norm"] and case["back"] else 4
        flops = 3 * n * case["pairs"] * 2 // case["head_dim"] + ((8 if case["back"] else 4) * n if case["norm"] else 0)
        more = 4 * case["tokens"] * case["axes"] + ((16 if case["back"] else 8) * case["head_dim"] if case["norm"] else 0)
        return {"bytes": moved * n + more, "flops": flops}
    lengths = _lengths(case)
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "step":
        t = sum(lengths)
        return {"bytes": 2 * (2 * t * hk * d + 2 * case["images"] * hq * d), "flops": 4 * t * hq * d}
    seen = 0
    for n in lengths:
        if case["mask"] == "document":
            seen += n * n
        else:
            p = (n * 2 + 4) // 5 if case["mask"] == "prefix" else 0
            seen += n * (n + 1) // 2 + p * (p - 1) // 2
    t = sum(lengths)
    # forward: two products; the gradients: five
    flops = 2 * seen * hq * d * (7 if case["train"] else 2)
    size = 2 * t * d * (2 * hq + 2 * hk)
    if case["train"]:
        size += 2 * t * d * (hq + hq + 2 * hk)
    return {"bytes": size, "flops": flops}
