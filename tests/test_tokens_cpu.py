"""Host side of the operators on packed patch tokens: what every call refuses, before anything touches a
GPU, the sizes of workspaces, and the plain forms that the GPU tests compare with.

The calls check their arguments ahead of the first HIP call, so they are made here with a stand-in for the
context (zeroed memory) and made-up device addresses: a refusal comes back as such, and what
is accepted ends in L3_ERR_DEVICE for want of a GPU.  (On a machine with one, accepted calls are not made.)"""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2208_08711_amd as l3
import token_refs as ref
from paper_2208_08711_amd import binding as b

OK, INVALID, DEVICE, LIMIT = 0, 1, 7, 8
A = 0x10000                                     # an aligned address nobody reads
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def lib():
    return b._load()


_room = ctypes.create_string_buffer(1 << 16)
CTX = ctypes.addressof(_room)


def heads(d=A, token=512, head=64):
    return b._Heads(d, token, head)


def outcome(call, args, accepted):
    if accepted and torch.cuda.is_available():
        pytest.skip("accepted calls are for machines without a GPU")
    return call(*args)


def check(call, good, changes):
    """good: dict of arguments that are accepted; changes: (dict of changes, expected status)."""
    assert outcome(call, good.values(), True) == DEVICE
    for change, want in changes:
        args = {**good, **change}
        assert set(args) == set(good), change
        got = outcome(call, args.values(), want == DEVICE)
        assert got == want, (change, got)


# ---- patch tokens -------------------------------------------------------------------------------


def image(rgb=A + 1, stride=300, width=100, height=50):
    return (b._TokenImage * 1)(b._TokenImage(rgb, stride, width, height))


def three(*v):
    return (ctypes.c_float * 3)(*v)


def test_patch_tokens_refusals(lib):
    good = dict(ctx=CTX, images=image(), n=1, side=16, mean=three(0, 0, 0), stdv=three(1, 1, 1), dtype=0, d_tokens=A, tokens=28,
                d_positions=A, d_first=A, stream=None)
    check(lib.l3_patch_tokens_batch, good, [
        (dict(ctx=None), INVALID), (dict(images=None), INVALID), (dict(n=-1), INVALID), (dict(side=0), INVALID), (dict(side=65), INVALID),
        (dict(mean=None), INVALID), (dict(stdv=None), INVALID), (dict(stdv=three(1, 0, 1)), INVALID), (dict(dtype=2), INVALID),
        (dict(d_tokens=None), INVALID), (dict(d_tokens=A + 8), INVALID), (dict(tokens=27), INVALID), (dict(tokens=-1), INVALID),
        (dict(d_positions=A + 2), INVALID), (dict(d_first=A + 1), INVALID),
        (dict(images=image(rgb=None)), INVALID), (dict(images=image(stride=299)), INVALID), (dict(images=image(width=0)), INVALID),
        (dict(images=image(height=0)), INVALID),
        (dict(images=image(stride=3 << 32, width=0xFFFFFFFF, height=0xFFFFFFFF), tokens=1 << 60), LIMIT),
        (dict(images=image(stride=3 << 17, width=1 << 17, height=1 << 14), side=1, tokens=1 << 31), LIMIT),
        (dict(images=image(stride=3 << 28, width=1 << 28, height=1), side=64, tokens=1 << 22), LIMIT),
        (dict(images=image(height=1 << 28), side=64, tokens=1 << 23), LIMIT), (dict(n=0, tokens=0), OK), (dict(n=0, images=None, tokens=0, d_tokens=None), OK), (dict(d_positions=None, d_first=None), DEVICE)])


def test_patch_tokens_count():
    for w, h, side in ((1, 1, 1), (100, 50, 16), (64, 64, 64), (65, 64, 64), (0xFFFFFFFF, 3, 2)):
        assert l3.patch_tokens_count(w, h, side) == -(-w // side) * -(-h // side)
    for w, h, side in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 65)):
        assert l3.patch_tokens_count(w, h, side) == 0


# ---- dropout ------------------------------------------------------------------------------------


def test_dropout_refusals(lib):
    good = dict(ctx=CTX, x=A, xs=64, r=A, rs=64, y=A, ys=64, rows=4, cols=64, dtype=1, p=0.5, seed=1, offset=2, d_offset=A, stream=None)
    check(lib.l3_dropout, good, [
        (dict(ctx=None), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x=A + 1), INVALID), (dict(y=A + 1), INVALID),
        (dict(r=A + 1), INVALID), (dict(d_offset=A + 4), INVALID), (dict(xs=63), INVALID), (dict(ys=63), INVALID), (dict(rs=63), INVALID),
        (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(dtype=-1), INVALID), (dict(dtype=2), INVALID), (dict(p=-0.01), INVALID),
        (dict(p=1.01), INVALID), (dict(p=NAN), INVALID), (dict(rows=1 << 40, cols=1 << 40, xs=1 << 40, ys=1 << 40, rs=1 << 40), LIMIT),
        (dict(rows=0, x=None), OK), (dict(cols=0, y=None), OK), (dict(r=None, rs=0, d_offset=None), DEVICE), (dict(p=1.0), DEVICE)])


def test_generator_known_answers():
    """The round function of the plain form, at ten rounds, against the known answers that its authors publish with
    their generator (all zeros, all ones, digits of pi), so that the seven-round masks rest on the same rounds."""
    ones, pi = 0xFFFFFFFF, (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344, 0xA4093822, 0x299F31D0)
    for c, k, want in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                       ((ones,) * 4, (ones,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                       (pi[:4], pi[4:], (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = ref.philox(np.array([c[0] | c[1] << 32], dtype=np.uint64), c[2] | c[3] << 32, k[0] | k[1] << 32, rounds=10)
        assert got[0].tolist() == list(want)


def test_generator_shares():
    """Shares of elements that stay: over 2^20 elements off by at most five standard deviations."""
    n = 1 << 20
    for p in (0.1, 0.5, 0.9):
        assert abs(float(ref.kept(n, p, 5, 6).double().mean()) - (1 - p)) < 5 * math.sqrt(p * (1 - p) / n) + 2.0 ** -17


# ---- positions and norms ------------------------------------------------------------------------


def rotation(pairs=32, axes=1, magnitude=1.0, turns=True, positions=A):
    table = (ctypes.c_uint64 * 64)(*range(64))
    r = b._Rotation(pairs, axes, 0, magnitude, table if turns else None, positions)
    r.keep = table
    return r


BAD_ROTATIONS = ((dict(pairs=33), INVALID), (dict(pairs=-1), INVALID), (dict(axes=0), INVALID), (dict(axes=3), INVALID),
                 (dict(pairs=31, axes=2), INVALID), (dict(magnitude=INF), INVALID), (dict(magnitude=NAN), INVALID), (dict(turns=False), INVALID),
                 (dict(positions=None), INVALID), (dict(pairs=0, turns=False, positions=None), DEVICE), (dict(pairs=31), DEVICE))


def bad_heads(name):
    return [({name: heads(d=None)}, INVALID), ({name: heads(d=A + 1)}, INVALID), ({name: heads(token=-64)}, INVALID), ({name: heads(head=-64)}, INVALID)]


def test_rotate_refusals(lib):
    good = dict(ctx=CTX, rotation=rotation(), inverse=0, tokens=5, head_dim=64, q_heads=4, q=heads(), qo=heads(), k_heads=2, k=heads(), ko=heads(),
                dtype=0, stream=None)
    check(lib.l3_rotate, good, [(dict(rotation=rotation(**c)), want) for c, want in BAD_ROTATIONS] + [
        (dict(ctx=None), INVALID), (dict(rotation=None), INVALID), (dict(tokens=-1), INVALID), (dict(head_dim=63), INVALID), (dict(head_dim=0), INVALID),
        (dict(head_dim=130), INVALID), (dict(q_heads=-1), INVALID), (dict(k_heads=-1), INVALID), (dict(dtype=2), INVALID),
        (dict(tokens=1 << 31), LIMIT), (dict(q_heads=1025), LIMIT), (dict(k_heads=1025), LIMIT), (dict(tokens=0, q=heads(d=None)), OK),
        (dict(q_heads=0, k_heads=0), OK), (dict(k_heads=0, k=heads(d=None), ko=heads(d=None)), DEVICE)] +
        bad_heads("q") + bad_heads("qo") + bad_heads("k") + bad_heads("ko"))


def test_norm_rotate_refusals(lib):
    good = dict(ctx=CTX, rotation=rotation(), eps=1e-6, tokens=5, head_dim=64, q_heads=4, q=heads(), qw=A, qo=heads(), k_heads=2, k=heads(), kw=A,
                ko=heads(), dtype=1, stream=None)
    check(lib.l3_norm_rotate, good, [(dict(rotation=rotation(**c)), want) for c, want in BAD_ROTATIONS] + [
        (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(qw=None), INVALID), (dict(kw=None), INVALID),
        (dict(eps=0.0), DEVICE), (dict(k_heads=0, kw=None), DEVICE)] + bad_heads("q") + bad_heads("ko"))
    size = 1024 * 2 * 128 * 4
    good = dict(ctx=CTX, rotation=rotation(), eps=1e-6, tokens=5, head_dim=64, q_heads=4, q=heads(), qw=A, qg=heads(), qb=heads(), qwg=A, k_heads=2,
                k=heads(), kw=A, kg=heads(), kb=heads(), kwg=A, dtype=1, workspace=A, size=size, stream=None)
    check(lib.l3_norm_rotate_backward, good, [
        (dict(workspace=None), INVALID), (dict(workspace=A + 4), INVALID), (dict(size=size - 1), INVALID), (dict(qwg=None), INVALID),
        (dict(kwg=None), INVALID), (dict(qw=None), INVALID), (dict(q_heads=-1), INVALID), (dict(q_heads=0, k_heads=0), OK),
        (dict(q_heads=1025), LIMIT)] + bad_heads("qg") + bad_heads("kb") + bad_heads("qb"))


def test_rotation_table_refusals(lib):
    out = (ctypes.c_uint64 * 64)()
    good = dict(pairs=64, base=10000.0, factor=2.0, original=100.0, slow=1.0, fast=32.0, out=out)
    assert lib.l3_rotation_turns(*good.values()) == OK
    for change in (dict(pairs=0), dict(pairs=65), dict(base=1.0), dict(base=INF), dict(base=NAN), dict(factor=0.5), dict(factor=NAN), dict(original=-1.0),
                   dict(original=INF), dict(slow=32.0), dict(slow=NAN), dict(fast=INF), dict(out=None)):
        assert lib.l3_rotation_turns(*{**good, **change}.values()) == INVALID, change


# ---- attention ----------------------------------------------------------------------------------


def shape(**change):
    values = dict(head_dim=64, q_heads=4, kv_heads=2, images=3, q_tokens=100, kv_tokens=100, d_q_first=A, d_kv_first=None, mask=0, d_prefix=None,
                  scale=0.125, cap=0.0, d_slopes=None, dtype=0)
    assert not set(change) - set(values)
    return b._AttentionShape(*{**values, **change}.values())


BAD_SHAPES = [(dict(head_dim=60), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=136), INVALID), (dict(q_heads=3), INVALID),
              (dict(kv_heads=0), INVALID), (dict(q_heads=0), INVALID), (dict(images=-1), INVALID), (dict(q_tokens=-1), INVALID),
              (dict(kv_tokens=-1, d_kv_first=A), INVALID), (dict(kv_tokens=99), INVALID), (dict(d_q_first=None), INVALID),
              (dict(d_q_first=A + 2), INVALID), (dict(d_kv_first=A + 2), INVALID), (dict(mask=3), INVALID), (dict(mask=2), INVALID),
              (dict(mask=2, d_prefix=A + 1), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
              (dict(cap=-1.0), INVALID), (dict(cap=1e-44), INVALID), (dict(cap=NAN), INVALID), (dict(d_slopes=A + 2), INVALID), (dict(dtype=2), INVALID),
              (dict(q_tokens=1 << 31, kv_tokens=1 << 31), LIMIT), (dict(q_heads=65536, kv_heads=1), LIMIT)]
GOOD_SHAPES = [dict(mask=1), dict(mask=2, d_prefix=A), dict(cap=5.0), dict(d_slopes=A), dict(scale=0.0), dict(kv_tokens=7, d_kv_first=A), dict(head_dim=8)]


def bad_tiles(name):
    return [({name: heads(d=None)}, INVALID), ({name: heads(d=A + 8)}, INVALID), ({name: heads(token=-64)}, INVALID), ({name: heads(head=-64)}, INVALID),
            ({name: heads(token=516)}, INVALID), ({name: heads(head=68)}, INVALID)]


def test_attention_refusals(lib):
    good = dict(ctx=CTX, shape=shape(), q=heads(), k=heads(), v=heads(), out=heads(), lse=A, stream=None)
    check(lib.l3_attention, good, [(dict(shape=shape(**c)), want) for c, want in BAD_SHAPES] + [(dict(shape=shape(**c)), DEVICE) for c in GOOD_SHAPES] + [
        (dict(ctx=None), INVALID), (dict(shape=None), INVALID), (dict(lse=A + 2), INVALID), (dict(lse=None), DEVICE),
        (dict(shape=shape(images=0)), OK), (dict(shape=shape(q_tokens=0, kv_tokens=0, d_q_first=None), q=heads(d=None)), OK),
        (dict(shape=shape(kv_tokens=0, d_kv_first=A), k=heads(d=None), v=heads(d=None)), DEVICE), (dict(k=heads(token=1 << 24)), LIMIT)] +
        bad_tiles("q") + bad_tiles("k") + bad_tiles("v") + bad_tiles("out"))


def test_attention_backward_refusals(lib):
    size = lib.l3_attention_workspace(ctypes.byref(shape()))
    assert size >= 4 * 100 * 8
    good = dict(ctx=CTX, shape=shape(), q=heads(), k=heads(), v=heads(), out=heads(), lse=A, og=heads(), qg=heads(), kg=heads(), vg=heads(), workspace=A,
                size=size, stream=None)
    check(lib.l3_attention_backward, good, [(dict(shape=shape(**c)), want) for c, want in BAD_SHAPES] + [
        (dict(lse=None), INVALID), (dict(lse=A + 2), INVALID), (dict(workspace=None), INVALID), (dict(workspace=A + 8), INVALID),
        (dict(size=size - 1), INVALID), (dict(shape=shape(images=0)), OK), (dict(og=heads(token=1 << 24)), LIMIT)] +
        bad_tiles("q") + bad_tiles("og") + bad_tiles("qg") + bad_tiles("kg") + bad_tiles("vg"))
    for change, _ in BAD_SHAPES:
        assert lib.l3_attention_workspace(ctypes.byref(shape(**change))) == 0
    assert lib.l3_attention_workspace(None) == 0
    # a workspace never shrinks as tokens are added within one split, and large ones do not wrap
    assert lib.l3_attention_workspace(ctypes.byref(shape(q_tokens=(1 << 31) - (1 << 17), kv_tokens=(1 << 31) - (1 << 17), q_heads=64, kv_heads=64))) >= (1 << 31) * 63 * 8


def test_step_refusals(lib):
    size = lib.l3_attention_step_workspace(3, 64, 4, 2, 1000)
    good = dict(ctx=CTX, n=3, head_dim=64, q_heads=4, kv_heads=2, q=heads(), k=heads(), ks=64000, v=heads(), vs=64000, lengths=A, most=1000, scale=0.1,
                cap=0.0, slopes=None, out=heads(), dtype=0, workspace=A, size=size, stream=None)
    check(lib.l3_attention_step, good, [
        (dict(ctx=None), INVALID), (dict(n=-1), INVALID), (dict(head_dim=60), INVALID), (dict(q_heads=3), INVALID), (dict(kv_heads=0), INVALID),
        (dict(ks=-8), INVALID), (dict(vs=4), INVALID), (dict(lengths=None), INVALID), (dict(lengths=A + 2), INVALID), (dict(most=-1), INVALID),
        (dict(scale=-1.0), INVALID), (dict(cap=INF), INVALID), (dict(slopes=A + 1), INVALID), (dict(dtype=3), INVALID), (dict(workspace=None), INVALID),
        (dict(workspace=A + 8), INVALID), (dict(size=size - 1), INVALID), (dict(most=1 << 31), LIMIT), (dict(q_heads=65538), LIMIT), (dict(n=0), OK),
        (dict(k=heads(token=1 << 24)), LIMIT), (dict(slopes=A, cap=3.0), DEVICE), (dict(most=0, k=heads(d=None), v=heads(d=None)), DEVICE)] +
        bad_tiles("q") + bad_tiles("k") + bad_tiles("v") + bad_tiles("out"))
    for args in ((-1, 64, 4, 2, 10), (1, 60, 4, 2, 10), (1, 64, 3, 2, 10), (1, 64, 4, 2, -1), (1, 64, 4, 2, 1 << 31)):
        assert lib.l3_attention_step_workspace(*args) == 0


def test_binding_workspaces(lib):
    assert l3.attention_workspace(3, 100, 100, 4, 2, 64) == lib.l3_attention_workspace(ctypes.byref(shape()))
    assert l3.attention_step_workspace(3, 64, 4, 2, 1000) == lib.l3_attention_step_workspace(3, 64, 4, 2, 1000) > 0
    for call in (lambda: l3.attention_workspace(3, 100, 100, 4, 3, 64), lambda: l3.attention_step_workspace(3, 60, 4, 2, 10)):
        with pytest.raises(ValueError):
            call()


def test_binding_checks_tensors():
    """What the library cannot see, the binding checks: types, shapes, devices (here: that they are on a GPU)."""
    half, single = torch.zeros((4, 2, 64), dtype=torch.float16), torch.zeros((4, 2, 64))
    first = torch.zeros(2, dtype=torch.int32)

    class Ctx:
        handle = None

    for call in (lambda: l3.dropout(Ctx, half, half, 0.5, 1), lambda: l3.dropout(Ctx, single, single, 0.5, 1),
                 lambda: l3.rotate(Ctx, l3.Rotation([]), None, half, half), lambda: l3.attention(Ctx, half, half, half, half, first),
                 lambda: l3.attention_step(Ctx, half, half[None], half[None], first, half), lambda: l3.Rotation([0] * 65), lambda: l3.Rotation([0], axes=3)):
        with pytest.raises(ValueError):
            call()


# ---- the plain forms against others -------------------------------------------------------------


def test_plain_gradients_against_autograd():
    """The gradients of the plain forms, written from formulas, against torch's automatic ones in 64 bits."""
    gen = torch.Generator().manual_seed(1)
    x, w, g = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((5, 3, 8), (8,), (5, 3, 8)))
    x.requires_grad_(), w.requires_grad_()
    (ref.normed(x, w, 0.1) * g).sum().backward()
    gx, _, gw, _ = ref.norm_back(x.detach(), w.detach(), 0.1, g)
    assert torch.allclose(gx, x.grad, rtol=1e-12, atol=1e-13) and torch.allclose(gw, w.grad, rtol=1e-12, atol=1e-13)
    for mask, cap, slopes in ((0, 0.0, None), (1, 2.0, [0.5, 0.1]), (2, 0.0, [0.2, 0.3])):
        q, k, v, g = (torch.randn((9, h, 8), generator=gen, dtype=torch.float64).requires_grad_() for h in (2, 1, 1, 2))
        total = 0
        for a, e, pre in ((0, 4, 2), (4, 9, 9)):
            for h in range(2):
                s, _ = ref.scores(q[a:e, h], k[a:e, 0], mask, pre, 0.3, cap, slopes[h] if slopes else 0.0)
                total = total + (torch.softmax(s, -1) @ v[a:e, 0] * g[a:e, h].detach()).sum()
        total.backward()
        got = ref.attention(q, k, v, [0, 4, 9], [0, 4, 9], mask, [2, 9], 0.3, cap, slopes, torch.float16, g)
        for name, t in (("q_grad", q), ("k_grad", k), ("v_grad", v)):
            assert torch.allclose(got[name][0], t.grad, rtol=1e-10, atol=1e-12), (mask, name)
