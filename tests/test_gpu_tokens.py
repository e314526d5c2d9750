"""The operators on packed patch tokens (include/l3_tokens.h) on the GPU against their plain forms
in 64 bits (token_refs.py), at the sizes, layouts and masks where they can go wrong."""
import math

import numpy as np
import pytest

import oracle
import token_refs as ref
from paper_2208_08711_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = (torch.bfloat16, torch.float16)
MEAN, STDV = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)


@pytest.fixture(scope="module")
def l3():
    import paper_2208_08711_amd as l3
    assert torch.cuda.is_available(), "these tests need the GPU"
    return l3


@pytest.fixture(scope="module")
def ctx(l3):
    c = l3.Context(0)
    yield c
    c.close()


def normal(shape, seed, dtype, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def misaligned(t, by=1):
    """A copy that starts `by` elements behind an aligned address."""
    room = torch.empty(t.numel() + 8, dtype=t.dtype, device=t.device)[by:by + t.numel()].view(t.shape)
    room.copy_(t)
    return room


# ---- patch tokens -------------------------------------------------------------------------------


def want_tokens(l3, images, side, dtype):
    kind = l3.BF16 if dtype == torch.bfloat16 else l3.FP16
    table = l3.normalized_values(MEAN, STDV, kind)
    tokens, positions, first = [], [], [0]
    for im in images:
        h, w = im.shape[:2]
        rows, cols = -(-h // side), -(-w // side)
        planes = np.zeros((3, rows * side, cols * side), np.uint16)
        for c in range(3):
            planes[c, :h, :w] = table[c][im[:, :, c]]
        cut = planes.reshape(3, rows, side, cols, side).transpose(1, 3, 0, 2, 4)
        tokens.append(cut.reshape(rows * cols, -1))
        positions += [(r, c) for r in range(rows) for c in range(cols)]
        first.append(first[-1] + rows * cols)
    return np.concatenate(tokens), np.array(positions, np.int32), np.array(first, np.int32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("side", (1, 3, 7, 8, 14, 16, 33, 64))
def test_patch_tokens(l3, ctx, side, dtype):
    rng = np.random.default_rng(side)
    images = [rng.integers(0, 256, (h, w, 3), dtype=np.uint8) for h, w in ((1, 1), (64, 64), (33, 47), (5, 300), (130, 129), (16, 15))]
    want, positions, first = want_tokens(l3, images, side, dtype)
    # images at odd addresses, one with rows apart
    dev = [misaligned(torch.from_numpy(im).cuda(), k % 4) for k, im in enumerate(images)]
    apart = torch.full((images[2].shape[0], images[2].shape[1] + 5, 3), 7, dtype=torch.uint8, device="cuda")
    apart[:, :images[2].shape[1]] = dev[2]
    dev[2] = apart[:, :images[2].shape[1]]
    total = sum(l3.patch_tokens_count(im.shape[1], im.shape[0], side) for im in images)
    assert total == len(want)
    room = torch.full((total + 2, 3 * side * side), -3.0, dtype=dtype, device="cuda")
    at, starts = torch.full((total, 2), -1, dtype=torch.int32, device="cuda"), torch.full((len(images) + 1,), -1, dtype=torch.int32, device="cuda")
    l3.patch_tokens_batch(ctx, dev, side, MEAN, STDV, room[:total], positions=at, first=starts)
    got = room[:total].cpu().view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(got, want)
    assert np.array_equal(at.cpu().numpy(), positions) and np.array_equal(starts.cpu().numpy(), first)
    assert bool((room[total:] == -3.0).all()), "written behind the last token"


def test_patch_tokens_many_images_and_a_wide_one(l3, ctx):
    """More images than one launch's arguments hold, and rows of patches of many strips."""
    rng = np.random.default_rng(3)
    images = [rng.integers(0, 256, (int(h), int(w), 3), dtype=np.uint8) for h, w in rng.integers(1, 40, (150, 2))]
    images.append(rng.integers(0, 256, (40, 3001, 3), dtype=np.uint8))
    want, positions, first = want_tokens(l3, images, 8, torch.bfloat16)
    out = torch.empty((len(want), 192), dtype=torch.bfloat16, device="cuda")
    starts = torch.empty(len(images) + 1, dtype=torch.int32, device="cuda")
    l3.patch_tokens_batch(ctx, [torch.from_numpy(im).cuda() for im in images], 8, MEAN, STDV, out, first=starts)
    assert np.array_equal(out.cpu().view(torch.int16).numpy().view(np.uint16), want)
    assert np.array_equal(starts.cpu().numpy(), first)


# ---- dropout ------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", ((1, 1), (1, 7), (1, 8), (3, 5), (4, 64), (17, 129), (300, 1000)))
@pytest.mark.parametrize("layout", ("flat", "apart", "wide rows", "odd"))
@pytest.mark.parametrize("residual", (False, True))
def test_dropout(l3, ctx, rows, cols, layout, residual, dtype):
    p, seed, offset = 0.3, 0xFEDCBA9876543210, 2 ** 40 + 5
    x, z = normal((rows, cols), 1, dtype), normal((rows, cols), 2, dtype)
    x[0, 0] = math.nan
    out = torch.full((rows, cols), 9.0, dtype=dtype, device="cuda")
    guard = None
    if layout == "apart":
        wide = [torch.full((rows, cols + 3), 5.0, dtype=dtype, device="cuda") for _ in range(3)]
        wide[0][:, :cols], wide[1][:, :cols] = x, z
        x, z, out, guard = wide[0][:, :cols], wide[1][:, :cols], wide[2][:, :cols], wide[2][:, cols:]
    elif layout == "wide rows":                                         # aligned rows apart
        wide = [torch.full((rows, (cols + 15) // 8 * 8), 5.0, dtype=dtype, device="cuda") for _ in range(3)]
        wide[0][:, :cols], wide[1][:, :cols] = x, z
        x, z, out, guard = wide[0][:, :cols], wide[1][:, :cols], wide[2][:, :cols], wide[2][:, cols:]
    elif layout == "odd":
        x, z, out = misaligned(x), misaligned(z, 3), misaligned(out)
    l3.dropout(ctx, x, out, p, seed, offset=offset, residual=z if residual else None)
    keep = ref.kept(rows * cols, p, seed, offset).view(rows, cols)
    scale = 65536.0 / (65536 - int(p * 65536 + 0.5))
    want = torch.where(keep, x.cpu().double() * scale, 0.0)
    size = want.abs()
    if residual:
        want, size = want + z.cpu().double(), size + z.cpu().double().abs()
    got = out.cpu()
    assert bool((got[0, 0].isnan() == want[0, 0].isnan()))
    got[0, 0], want[0, 0], size[0, 0] = 0, 0, 0
    ref.close(got, want, 2.0 ** -22 * size, "dropout")
    if guard is not None:
        assert bool((guard == 5.0).all()), "written between the rows"


@pytest.mark.parametrize("p", (0.0, 1.0, 1e-9, 0.5, 1 - 2.0 ** -16))
def test_dropout_shares(l3, ctx, p):
    """The ends of the range, and in place; the share that stays is the generator's."""
    x = normal((64, 1024), 3, torch.bfloat16)
    want = x.cpu().double() * (65536.0 / max(1, 65536 - int(p * 65536 + 0.5))) * ref.kept(x.numel(), p, 7, 0).view(x.shape)
    l3.dropout(ctx, x, x, p, 7)
    ref.close(x, want, 2.0 ** -22 * want.abs(), "dropout")


def test_dropout_gradient_is_the_same_call(l3, ctx):
    """The derivative of y along any direction is the same mask and scale on it: linear, so a difference
    of two calls is it exactly but for roundings (none at p = 1/2 and powers of two)."""
    x, d = torch.ones((8, 96), dtype=torch.float16, device="cuda"), torch.full((8, 96), 2.0, dtype=torch.float16, device="cuda")
    y0, y1, g = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    z = normal((8, 96), 4, torch.float16) * 0
    l3.dropout(ctx, x, y0, 0.5, 11, offset=3, residual=z)
    l3.dropout(ctx, x + d, y1, 0.5, 11, offset=3, residual=z)
    l3.dropout(ctx, d, g, 0.5, 11, offset=3)
    assert torch.equal(y1 - y0, g)


# ---- positions and norms ------------------------------------------------------------------------

LAYOUTS = ((64, 32, 1, False), (64, 32, 2, True), (128, 64, 2, False), (128, 32, 1, True), (72, 36, 1, False), (80, 40, 2, True),
           (88, 22, 1, False), (32, 16, 2, False), (2, 1, 1, True), (6, 3, 1, False), (128, 0, 1, False), (10, 2, 2, False))


def table(l3, pairs, axes):
    return l3.rotation_turns(pairs // axes) * axes if pairs else []


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim,pairs,axes,interleaved", LAYOUTS)
@pytest.mark.parametrize("odd", (False, True))
@pytest.mark.parametrize("inverse", (False, True))
def test_rotate(l3, ctx, head_dim, pairs, axes, interleaved, odd, inverse, dtype):
    tokens, hq, hk = 37, 5, 2
    joint = normal((tokens, hq + 2 * hk, head_dim), 5, dtype)
    if odd:
        joint = misaligned(joint)
    q, k = joint[:, :hq], joint[:, hq:hq + hk]
    q_out, k_out = torch.empty((tokens, hq, head_dim), dtype=dtype, device="cuda"), torch.empty((hk, tokens, head_dim), dtype=dtype, device="cuda").transpose(0, 1)
    where = torch.randint(-5000, 1 << 20, (tokens, axes), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    where[0], where[1], where[2] = 0, 2 ** 31 - 1, -2 ** 31
    rotation = l3.Rotation(table(l3, pairs, axes), axes=axes, interleaved=interleaved, magnitude=1.25)
    l3.rotate(ctx, rotation, where.cuda(), q, q_out, k, k_out, inverse=inverse)
    angle = ref.angles(table(l3, pairs, axes), axes, where)
    for got, x in ((q_out, q), (k_out, k)):
        want, size = ref.turned(x.cpu().double(), angle, pairs, interleaved, 1.25, back=inverse)
        ref.close(got, want, ref.SLACK * size, "rotate")
        if 2 * pairs < head_dim:
            assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])
    before = q.clone()
    l3.rotate(ctx, rotation, where.cuda(), q, q, inverse=inverse)
    assert torch.equal(q, q_out) and torch.equal(joint[:, hq:], torch.cat((k, joint[:, hq + hk:]), 1)) and q.shape == before.shape


def test_rotation_tables(l3):
    """The table and its stretched forms against 64-bit arithmetic: some tens of roundings of 2^-53 in the check, below
    1e-13 together, and half a unit of the integer, which relative to an integer t is 0.5 / t (2e-13 at the lowest frequency here)."""
    for pairs, base, factor, original in ((32, 10000.0, 1.0, 0.0), (64, 500000.0, 8.0, 8192.0), (16, 100.0, 4.0, 0.0), (1, 10000.0, 2.0, 77.0)):
        got = l3.rotation_turns(pairs, base, factor=factor, original_length=original)
        for j, t in enumerate(got):
            f = base ** (-j / pairs)
            keep = 0.0
            if original:
                keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - 1) / 31))
            if factor > 1:
                f *= keep + (1 - keep) / factor
            assert abs(t / 2.0 ** 64 * 2 * math.pi / f - 1) < 1e-13 + 0.5 / t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim,pairs,axes,interleaved", LAYOUTS)
@pytest.mark.parametrize("odd", (False, True))
@pytest.mark.parametrize("tokens", (1, 67))
def test_norm_rotate_and_gradients(l3, ctx, head_dim, pairs, axes, interleaved, odd, tokens, dtype):
    hq, hk, eps, magnitude = 4, 3, 1e-3, 0.75
    joint = normal((tokens, hq + 2 * hk, head_dim), 7, dtype)
    joint[0, 0] = 0                                                       # a head of zeros: eps alone
    if odd:
        joint = misaligned(joint)
    q, k = joint[:, :hq], joint[:, hq:hq + hk]
    qw, kw = (1 + 0.3 * normal((head_dim,), 8 + i, torch.float32) for i in range(2))
    qg, kg = normal((tokens, hq, head_dim), 10, dtype), normal((tokens, hk, head_dim), 11, dtype)
    qo, ko, qb, kb = (torch.empty_like(t) for t in (qg, kg, qg, kg))
    qwg, kwg = torch.empty_like(qw), torch.empty_like(kw)
    where = torch.randint(0, 3000, (tokens, axes), generator=torch.Generator().manual_seed(12), dtype=torch.int32)
    rotation = l3.Rotation(table(l3, pairs, axes), axes=axes, interleaved=interleaved, magnitude=magnitude)
    l3.norm_rotate(ctx, rotation, where.cuda(), q, qw, qo, k, kw, ko, eps=eps)
    l3.norm_rotate_backward(ctx, rotation, where.cuda(), q, qw, qg, qb, qwg, k, kw, kg, kb, kwg, eps=eps)
    angle = ref.angles(table(l3, pairs, axes), axes, where)
    for x, w, g, o, b, wg in ((q, qw, qg, qo, qb, qwg), (k, kw, kg, ko, kb, kwg)):
        x, w, g = x.cpu().double(), w.cpu().double(), g.cpu().double()
        n = ref.normed(x, w, eps)
        want, size = ref.turned(n, angle, pairs, interleaved, magnitude)
        ref.close(o, want, ref.SLACK * size, "norm_rotate")
        back, back_size = ref.turned(g, angle, pairs, interleaved, magnitude, back=True)
        gx, gx_size, gw, gw_size = ref.norm_back(x, w, eps, back)
        _, most, _, most_w = ref.norm_back(x, w, eps, back_size)            # terms of the turned gradient, absolute
        ref.close(b, gx, ref.SLACK * torch.maximum(gx_size, most), "gradient of x")
        off = (wg.cpu().double() - gw).abs()
        assert bool((off <= 2 * ref.SLACK * torch.maximum(gw_size, ref.norm_back(x.abs(), w.abs(), eps, back_size)[2])).all()), off.max()
    # the same bits again, and in place of the gradients
    again = torch.empty_like(qwg)
    qg2, kg2 = qg.clone(), kg.clone()
    l3.norm_rotate_backward(ctx, rotation, where.cuda(), q, qw, qg2, qg2, again, k, kw, kg2, kg2, torch.empty_like(kwg), eps=eps)
    assert torch.equal(again, qwg) and torch.equal(qg2, qb) and torch.equal(kg2, kb)


def test_norm_rotate_gradient_by_differences(l3, ctx):
    """Directional derivative of sum(g * y) in 64 bits against the gradients returned: differences of the formula at
    +-h along a direction, h = 2^-12, off by some h^2 = 2^-24 of the value and the gradients' own roundings."""
    tokens, heads, d = 9, 3, 64
    x, g, w = normal((tokens, heads, d), 13, torch.float16), normal((tokens, heads, d), 14, torch.float16), 1 + 0.2 * normal((d,), 15, torch.float32)
    where = torch.arange(tokens, dtype=torch.int32)
    rotation = l3.Rotation(l3.rotation_turns(32))
    back, wg = torch.empty_like(x), torch.empty_like(w)
    l3.norm_rotate_backward(ctx, rotation, where.cuda(), x, w, g, back, wg, eps=1e-6)
    angle = ref.angles(l3.rotation_turns(32), 1, where)

    def loss(x, w):
        return float((ref.turned(ref.normed(x, w, 1e-6), angle, 32, False, 1.0)[0] * g.cpu().double()).sum())

    xd, wd = normal(x.shape, 16, torch.float32).cpu().double(), normal(w.shape, 17, torch.float32).cpu().double()
    x, w, h = x.cpu().double(), w.cpu().double(), 2.0 ** -12
    by_x, by_w = (loss(x + h * xd, w) - loss(x - h * xd, w)) / (2 * h), (loss(x, w + h * wd) - loss(x, w - h * wd)) / (2 * h)
    got_x, got_w = (back.cpu().double() * xd).sum(), (wg.cpu().double() * wd).sum()
    assert abs(by_x - got_x) <= ref.half(torch.float16) * (back.cpu().double() * xd).abs().sum() + 2.0 ** -20 * abs(by_x)
    assert abs(by_w - got_w) <= ref.SLACK * 8 * (wg.cpu().double() * wd).abs().sum()


@pytest.mark.parametrize("tokens,heads", ((5000, 3), (70000, 1)))
def test_norm_rotate_many_tokens(l3, ctx, tokens, heads):
    """More tokens than one round of the workgroups: results of a sample, and the weights' gradient of all."""
    d = 64
    x, g, w = normal((tokens, heads, d), 18, torch.bfloat16), normal((tokens, heads, d), 19, torch.bfloat16), 1 + 0.2 * normal((d,), 20, torch.float32)
    rotation = l3.Rotation([], axes=1)
    out, back, wg = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    l3.norm_rotate(ctx, rotation, None, x, w, out)
    l3.norm_rotate_backward(ctx, rotation, None, x, w, g, back, wg)
    xd, wd, gd = x.cpu().double(), w.cpu().double(), g.cpu().double()
    ref.close(out, ref.normed(xd, wd, 1e-6), ref.SLACK * ref.normed(xd, wd, 1e-6).abs(), "norm")
    gx, gx_size, gw, gw_size = ref.norm_back(xd, wd, 1e-6, gd)
    ref.close(back, gx, ref.SLACK * gx_size, "gradient of x")
    assert bool(((wg.cpu().double() - gw).abs() <= ref.SLACK * gw_size).all())


@pytest.mark.parametrize("heads", ((1001, 1), (13, 1024), (0, 7)))
def test_norm_rotate_many_heads(l3, ctx, heads):
    """More heads than one workgroup, or all of them, have slots for; and no queries at all."""
    hq, hk = heads
    tokens, d = 150, 8
    x, g = [normal((tokens, h, d), 80 + h, torch.bfloat16) for h in heads], [normal((tokens, h, d), 81 + h, torch.bfloat16) for h in heads]
    w = [1 + 0.2 * normal((d,), 82 + i, torch.float32) for i in range(2)]
    rotation, where = l3.Rotation(l3.rotation_turns(4)), torch.arange(tokens, dtype=torch.int32)
    out, back, wg = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in x], [torch.full_like(t, 5.0) for t in w]
    l3.norm_rotate(ctx, rotation, where.cuda(), x[0], w[0], out[0], x[1], w[1], out[1])
    l3.norm_rotate_backward(ctx, rotation, where.cuda(), x[0], w[0], g[0], back[0], wg[0], x[1], w[1], g[1], back[1], wg[1])
    angle = ref.angles(l3.rotation_turns(4), 1, where)
    for i in range(2):
        if not heads[i]:
            continue
        xd, wd, gd = x[i].cpu().double(), w[i].cpu().double(), g[i].cpu().double()
        want, size = ref.turned(ref.normed(xd, wd, 1e-6), angle, 4, False, 1.0)
        ref.close(out[i], want, ref.SLACK * size, "norm_rotate")
        turned, most = ref.turned(gd, angle, 4, False, 1.0, back=True)
        gx, gx_size, gw, _ = ref.norm_back(xd, wd, 1e-6, turned)
        _, big, _, gw_size = ref.norm_back(xd, wd, 1e-6, most)
        ref.close(back[i], gx, ref.SLACK * torch.maximum(gx_size, big), "gradient of x")
        assert bool(((wg[i].cpu().double() - gw).abs() <= ref.SLACK * gw_size).all())


# ---- attention ----------------------------------------------------------------------------------


def first_of(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def run_attention(l3, ctx, lengths, kv_lengths, heads, head_dim, dtype, mask, cap, slopes, behind=5, seed=21):
    """Forward and gradients against the plain form; tokens behind the last image hold NaN and stay as they are."""
    q_first, kv_first = first_of(lengths), first_of(kv_lengths if kv_lengths is not None else lengths)
    tq, tk = q_first[-1] + behind, kv_first[-1] + behind
    hq, hk = heads
    if kv_lengths is None:
        joint = normal((tq, hq + 2 * hk, head_dim), seed, dtype)
        joint[q_first[-1]:] = math.nan
        q, k, v = joint[:, :hq], joint[:, hq:hq + hk], joint[:, hq + hk:]
    else:                                                                # head-major memory
        q = normal((hq, tq, head_dim), seed, dtype).transpose(0, 1)
        k, v = (normal((hk, tk, head_dim), seed + i, dtype).transpose(0, 1) for i in (1, 2))
        q[q_first[-1]:], k[kv_first[-1]:], v[kv_first[-1]:] = math.nan, math.nan, math.nan
    grad = normal((tq, hq, head_dim), seed + 3, dtype)
    grad[q_first[-1]:] = math.nan
    prefix = [(3 * n) // 4 if i % 2 else n + 9 for i, n in enumerate(kv_lengths or lengths)] if mask == l3.MASK_PREFIX else None
    steep = [2.0 ** -(h + 1) for h in range(hq)] if slopes else None
    how = dict(mask=mask, cap=cap, scale=head_dim ** -0.5,
               kv_first=None if kv_lengths is None else torch.tensor(kv_first, dtype=torch.int32, device="cuda"),
               prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda"),
               slopes=None if steep is None else torch.tensor(steep, device="cuda"))
    table = torch.tensor(q_first, dtype=torch.int32, device="cuda")
    out = torch.full((tq, hq, head_dim), 3.0, dtype=dtype, device="cuda")
    lse = torch.full((hq, tq), 3.0, device="cuda")
    l3.attention(ctx, q, k, v, out, table, lse=lse, **how)
    want = ref.attention(q, k, v, q_first, kv_first, mask, prefix, head_dim ** -0.5, cap, steep, dtype, grad)
    n, m = q_first[-1], kv_first[-1]
    ref.close(out[:n], want["out"][0][:n], want["out"][1][:n], "out")
    assert bool((out[n:] == 3.0).all()) and bool((lse[:, n:] == 3.0).all()), "written behind the last image"
    got, at = lse[:, :n].cpu().double(), want["lse"][0][:, :n]
    assert torch.equal(got == -math.inf, at == -math.inf)
    some = at > -math.inf
    assert bool(((got - at).abs() <= want["lse"][1][:, :n])[some].all()), "lse"
    grads = [torch.full(t.shape, 3.0, dtype=dtype, device="cuda") for t in (q, k, v)]
    l3.attention_backward(ctx, q, k, v, out, lse, grad, *grads, table, **how)
    for name, got, end in zip(("q_grad", "k_grad", "v_grad"), grads, (n, m, m)):
        ref.close(got[:end], want[name][0][:end], want[name][1][:end], name)
        assert bool((got[end:] == 3.0).all()), "written behind the last image"
    # the same call gives the same bits
    again = [torch.empty_like(t) for t in grads]
    l3.attention_backward(ctx, q, k, v, out, lse, grad, *again, table, **how)
    for a, b, end in zip(again, grads, (n, m, m)):
        assert torch.equal(a[:end], b[:end])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", (0, 1, 2))
@pytest.mark.parametrize("head_dim", (8, 32, 64, 72, 96, 128))
def test_attention_widths_and_masks(l3, ctx, head_dim, mask, dtype):
    run_attention(l3, ctx, (1, 0, 63, 130, 2), None, (4, 2), head_dim, dtype, mask, 0.0, False)


@pytest.mark.parametrize("mask", (0, 1, 2))
@pytest.mark.parametrize("cap,slopes", ((0.0, True), (2.0, False), (20.0, True)))
@pytest.mark.parametrize("head_dim,dtype", ((40, torch.bfloat16), (64, torch.float16), (88, torch.bfloat16), (128, torch.float16)))
def test_attention_capped_and_biased(l3, ctx, head_dim, dtype, cap, slopes, mask):
    run_attention(l3, ctx, (65, 7, 200), None, (3, 1), head_dim, dtype, mask, cap, slopes)


@pytest.mark.parametrize("mask", (0, 1, 2))
@pytest.mark.parametrize("head_dim,dtype", ((64, torch.bfloat16), (128, torch.bfloat16), (24, torch.float16)))
def test_attention_more_or_fewer_keys(l3, ctx, head_dim, dtype, mask):
    """Queries that see nothing: more queries than keys, images without keys or queries."""
    run_attention(l3, ctx, (5, 100, 0, 129, 3, 64), (77, 40, 9, 0, 1, 200), (2, 2), head_dim, dtype, mask, 0.0, mask == 1)


@pytest.mark.parametrize("lengths", ((128,), (129,), (257, 255), (640,), tuple([1] * 130), tuple(range(70)), tuple(k % 5 for k in range(1300)), tuple(k % 2 for k in range(4500))))
def test_attention_lengths(l3, ctx, lengths):
    """Ends of tiles, many images (more than one look at the table), and sums over many tiles."""
    run_attention(l3, ctx, lengths, None, (2, 1), 64, torch.bfloat16, 1, 0.0, False, behind=1 + len(lengths) % 3)
    run_attention(l3, ctx, lengths, None, (1, 1), 128, torch.float16, 0, 0.0, False, behind=0)


@pytest.mark.parametrize("mask", (0, 1, 2))
@pytest.mark.parametrize("heads,head_dim,dtype", (((2, 2), 64, torch.bfloat16), ((4, 1), 128, torch.float16)))
def test_attention_long_images_and_few_heads(l3, ctx, heads, head_dim, dtype, mask):
    """Gradients whose keys and queries are shared out among workgroups, with images too short for that beside
    long ones; forward calls whose waves share the keys."""
    run_attention(l3, ctx, (1500, 3, 0, 700, 131), None, heads, head_dim, dtype, mask, 0.0, False)
    run_attention(l3, ctx, (2100, 40), (1100, 1900), heads, head_dim, dtype, mask, 0.0, False)


def test_attention_scores_far_apart(l3, ctx):
    """Scores that grow along the keys by far more than the reference point may lag, and large negative ones."""
    n, d = 300, 64
    k = torch.zeros((n, 1, d), dtype=torch.float16)
    k[:, 0, 0] = torch.linspace(-60, 60, n)
    q = torch.zeros((n, 1, d), dtype=torch.float16)
    q[:, 0, 0] = torch.linspace(-40, 40, n)
    v = normal((n, 1, d), 30, torch.float16)
    q, k = q.cuda(), k.cuda()
    out = torch.empty_like(q)
    l3.attention(ctx, q, k, v, out, torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale=1.0)
    want = ref.attention(q, k, v, [0, n], [0, n], 0, None, 1.0, 0.0, None, torch.float16)
    # products of up to 2400 are exact to 2^-13: exponents off by 2^-13 + 2^-12 (their product with log2 e)
    ref.close(out, want["out"][0], want["out"][1] + 2.0 ** -10 * v.abs().max().item(), "out")


def test_attention_infinities(l3, ctx):
    """A key whose score is -infinity has no weight; NaN in a query reaches its own row alone; an infinite value of
    another image reaches none."""
    d, table = 64, torch.tensor([0, 50, 100], dtype=torch.int32, device="cuda")
    q, k, v = normal((100, 1, d), 31, torch.bfloat16).abs(), normal((100, 1, d), 32, torch.bfloat16), normal((100, 1, d), 33, torch.bfloat16)
    k[7, 0, 3] = -math.inf
    q[20] = math.nan
    v[60, 0, 5] = math.inf
    out = torch.empty_like(q)
    l3.attention(ctx, q, k, v, out, table)
    keep = [i for i in range(50) if i != 20]
    others = [i for i in range(50) if i != 7]
    w = torch.softmax(q[keep, 0].cpu().double() @ k[others, 0].cpu().double().t() * d ** -0.5, -1)
    want = w @ v[others, 0].cpu().double()
    ref.close(out[keep, 0], want, (ref.half(torch.bfloat16) + 2 * ref.SLACK) * (w @ v[others, 0].cpu().double().abs()), "out")
    assert bool(out[20].isnan().all())
    assert bool((out[50:, 0, 5] == math.inf).all()) and bool(out[50:, 0, :5].isfinite().all()) and bool(out[50:, 0, 6:].isfinite().all())


def test_attention_without_keys_or_queries(l3, ctx):
    """No keys at all: zeros, and no gradient for the queries; no queries at all: none for keys and values."""
    some, none = normal((40, 2, 64), 36, torch.bfloat16), torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    a, z = torch.tensor([0, 40], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse, grads = torch.full_like(some, 3.0), torch.full((2, 40), 3.0, device="cuda"), torch.full_like(some, 3.0)
    l3.attention(ctx, some, none, none, out, a, kv_first=z, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    l3.attention_backward(ctx, some, none, none, out, lse, some, grads, none.clone(), none.clone(), a, kv_first=z)
    assert bool((grads == 0).all())
    k_grad, v_grad, empty = torch.full_like(some, 3.0), torch.full_like(some, 3.0), torch.empty((2, 0), device="cuda")
    l3.attention(ctx, none, some, some, none.clone(), z, kv_first=a, lse=empty)
    l3.attention_backward(ctx, none, some, some, none, empty, none, none.clone(), k_grad, v_grad, z, kv_first=a)
    assert bool((k_grad == 0).all()) and bool((v_grad == 0).all())


def test_attention_scale_of_zero(l3, ctx):
    """Weights are all alike."""
    q, k, v = (normal((70, 1, 32), 34 + i, torch.bfloat16) for i in range(3))
    out = torch.empty_like(q)
    l3.attention(ctx, q, k, v, out, torch.tensor([0, 70], dtype=torch.int32, device="cuda"), scale=0.0, mask=l3.MASK_CAUSAL)
    want = v.cpu().double().cumsum(0) / torch.arange(1, 71)[:, None, None]
    size = v.cpu().double().abs().cumsum(0) / torch.arange(1, 71)[:, None, None]
    ref.close(out, want, ref.SLACK * size, "out")


def test_attention_gradient_by_differences(l3, ctx):
    """Directional derivative of sum(g * out) in 64 bits by differences, against the gradients returned."""
    lengths, d, dtype = (40, 33), 32, torch.float16
    first = first_of(lengths)
    q, k, v, g = (normal((73, h, d), 40 + i, dtype) for i, h in enumerate((4, 2, 2, 4)))
    table = torch.tensor(first, dtype=torch.int32, device="cuda")
    steep = [0.5, 0.25, 0.125, 0.0625]
    how = dict(mask=l3.MASK_CAUSAL, cap=3.0, slopes=torch.tensor(steep, device="cuda"), scale=0.2)
    out, lse = torch.empty_like(q), torch.empty((4, 73), device="cuda")
    l3.attention(ctx, q, k, v, out, table, lse=lse, **how)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    l3.attention_backward(ctx, q, k, v, out, lse, g, *grads, table, **how)
    tensors, g = [t.cpu().double() for t in (q, k, v)], g.cpu().double()

    def loss(tensors):
        return float((ref.attention(*tensors, first, first, 1, None, 0.2, 3.0, steep, dtype)["out"][0] * g).sum())

    want = ref.attention(*tensors, first, first, 1, None, 0.2, 3.0, steep, dtype, g)
    for i, name in enumerate(("q_grad", "k_grad", "v_grad")):
        direction, h = normal(tensors[i].shape, 50 + i, torch.float32).cpu().double(), 2.0 ** -11
        ends = []
        for sign in (1, -1):
            moved = list(tensors)
            moved[i] = tensors[i] + sign * h * direction
            ends.append(loss(moved))
        by = (ends[0] - ends[1]) / (2 * h)
        got = float((grads[i].cpu().double() * direction).sum())
        room = float(((want[name][1] + ref.half(dtype) * want[name][0].abs()) * direction.abs()).sum())
        # central differences: h^2/6 of the third derivative, which for these sizes stays below 2^-14 of the size of the terms
        assert abs(by - got) <= room + 2.0 ** -14 * float((want[name][0] * direction).abs().sum()), name


# ---- single tokens ------------------------------------------------------------------------------


def run_step(l3, ctx, lengths, room, heads, head_dim, dtype, cap, slopes, seed=60, head_major=False, max_length=None):
    n, (hq, hk) = len(lengths), heads
    q = normal((n, hq, head_dim), seed, dtype)
    caches = []
    for i in (1, 2):
        c = normal((n, hk, room, head_dim) if head_major else (n, room, hk, head_dim), seed + i, dtype)
        caches.append(c.transpose(1, 2) if head_major else c)
    for b, m in enumerate(lengths):
        for c in caches:
            c[b, m:] = math.nan
    steep = [2.0 ** -(h % 8 + 1) for h in range(hq)] if slopes else None
    out = torch.full_like(q, 3.0)
    l3.attention_step(ctx, q, *caches, torch.tensor(lengths, dtype=torch.int32, device="cuda"), out, cap=cap, max_length=max_length,
                      slopes=None if steep is None else torch.tensor(steep, device="cuda"))
    for b, m in enumerate(lengths):
        k, v = caches[0][b, :m], caches[1][b, :m]
        want = ref.attention(q[b:b + 1], k, v, [0, 1], [0, m], 1, None, head_dim ** -0.5, cap, steep, dtype)
        ref.close(out[b:b + 1], want["out"][0], want["out"][1], "sequence %d" % b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim", (8, 32, 64, 80, 128))
@pytest.mark.parametrize("heads", ((1, 1), (6, 2), (32, 1), (40, 1)))
def test_step(l3, ctx, heads, head_dim, dtype):
    run_step(l3, ctx, (0, 1, 31, 32, 33, 64, 65, 257, 500), 500, heads, head_dim, dtype, 0.0, False)


@pytest.mark.parametrize("cap,slopes", ((0.0, True), (3.0, False), (30.0, True)))
@pytest.mark.parametrize("head_dim", (64, 96, 128))
def test_step_capped_and_biased(l3, ctx, head_dim, cap, slopes):
    run_step(l3, ctx, (700, 3, 0), 701, (8, 2), head_dim, torch.bfloat16, cap, slopes, head_major=True)


def test_step_long(l3, ctx):
    """Many pieces of one cache, and one that is far shorter than the room says."""
    run_step(l3, ctx, (20011, 130, 1), 20011, (2, 1), 64, torch.float16, 0.0, False)
    run_step(l3, ctx, (40,), 60000, (2, 1), 128, torch.bfloat16, 0.0, False)
    run_step(l3, ctx, (100, 17), 4096, (4, 4), 128, torch.bfloat16, 0.0, False, max_length=100)
