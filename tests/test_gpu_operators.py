"""Rotary positions and rows in 8 bits on the GPU, through the C ABI, against the plain evaluations in tests/operators_ref.py."""
import ctypes

import numpy as np
import pytest
import torch

import operators_ref as ref
import paper_2503_09387_amd as vs
from gpu_util import DEV, check_close, lens_array, scale32, vs_shape
from synth import AttnShape, to_f64

pytestmark = pytest.mark.gpu

HEADS = [(28, 4), (8, 8), (8, 1), (12, 6), (5, 5), (6, 3)]


@pytest.fixture(autouse=True)
def _reset_tuning():
    yield
    for knob in (0, 1, 2, 4):
        vs.set_tuning(knob, 0)


def rows(seed, *dims, loud=True, sigma=0.5):
    """K or V rows [..][128] on the GPU: some channels several times the others, rows of different sizes."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(dims, generator=g, device=DEV) * sigma
    if loud:
        x *= 1 + 7 * (torch.rand(dims[-2:], generator=g, device=DEV) < 0.03)
        x *= torch.exp2(torch.randint(-3, 4, dims[:-1] + (1,), generator=g, device=DEV).float())
    return x.to(torch.bfloat16)


def f64(t):
    return t.double().cpu().numpy()


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def slab_of(shape, n, capacity, fill=0xFF):
    """Memory that holds something else: scales of it are not numbers."""
    return torch.full((n, vs.cache8_bytes(shape, capacity)), fill, dtype=torch.uint8, device=DEV)


def held(x):
    """What rows read back as: the exact product of the whole number and the scale, rounded to bf16."""
    return torch.from_numpy(ref.stands_for(f64(x)).astype(np.float32)).to(torch.bfloat16)


def off_by(out, want):
    """What the values are off; a value past the largest bf16 by less than half a step is an infinity when it is rounded."""
    got = f64(out)
    most = float(torch.finfo(torch.bfloat16).max)
    got = np.where(np.isinf(got) & (np.abs(want) >= most * (1 - 2.0 ** -9)), np.sign(got) * most, got)
    return np.where(np.isfinite(got), np.abs(got - want), np.inf)


# ---------------------------------------------------------------------------- rotary positions
def rotary_bound(x, ref_y, pos, dtype):
    """The revolutions are off by 3 roundings of 2^-53 of themselves (rate, product, 2 pi) and, in fp32, by 2^-26: an angle by 2 pi times
    that; sincospif is good to 4 ulp (2^-22); two products and a sum are 3 roundings of at most 2^-24 (|a| + |b|).  On top the
    output's own rounding."""
    reach = np.abs(x).max(-1, keepdims=True) * 2.0
    turns = np.abs(pos.astype(np.float64)).max() / (2 * np.pi)
    angle = 2 * np.pi * (2.0 ** -26 + 3 * 2.0 ** -53 * turns)
    eps = torch.finfo(dtype).eps / 2
    return reach * (angle + 2.0 ** -22 + 3 * 2.0 ** -24) * (1 + eps) + eps * np.abs(ref_y)


@pytest.mark.parametrize("dtype,dim,sections,pairing,inverse", [
    (torch.bfloat16, 128, (16, 24, 24), 0, False), (torch.bfloat16, 128, (16, 24, 24), 1, True), (torch.bfloat16, 128, (3, 0, 5), 0, True),
    (torch.bfloat16, 128, (1, 20, 11), 1, False), (torch.bfloat16, 128, (0, 0, 64), 0, False), (torch.float32, 64, (8, 12, 12), 0, False),
    (torch.float32, 64, (5, 2, 1), 1, True), (torch.float32, 64, (0, 24, 0), 0, True), (torch.float32, 128, (16, 24, 24), 0, False),
    (torch.float32, 128, (40, 7, 9), 1, False)])
@pytest.mark.parametrize("tokens,hq,hkv", [(1, 28, 4), (170, 28, 4), (37, 5, 5), (3, 64, 64), (300, 8, 1)])
def test_rotary(dtype, dim, sections, pairing, inverse, tokens, hq, hkv):
    sh = vs.Shape.make(hq, hkv, dim, "f32" if dtype == torch.float32 else "bf16")
    plan = vs.RotaryPlan(dim, sections, 1e6, pairing)
    g = torch.Generator(device=DEV).manual_seed(tokens + dim)
    q, k = (torch.randn((tokens, h, dim), generator=g, device=DEV).to(dtype) for h in (hq, hkv))
    pos = torch.randint(-2 ** 18, 2 ** 18, (3, tokens), generator=g, device=DEV, dtype=torch.int32)
    pos[:, 0] = torch.tensor([0, 2 ** 31 - 1, -2 ** 31])
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    vs.rotary(sh, plan, pos, q, k, qo, ko, inverse=inverse)
    for x, y in ((q, qo), (k, ko)):
        want = ref.rotate(f64(x), pos.cpu().numpy(), sections, 1e6, pairing == 0, inverse)
        err = np.abs(f64(y) - want)
        assert (err <= rotary_bound(f64(x), want, pos.cpu().numpy(), dtype)).all(), err.max()
        n = 2 * sum(sections)
        assert same_bits(y[..., n:], x[..., n:])
    # in place, and one of the two alone
    qi, ki = q.clone(), k.clone()
    vs.rotary(sh, plan, pos, qi, ki, qi, ki, inverse=inverse)
    assert same_bits(qi, qo) and same_bits(ki, ko)
    alone = torch.empty_like(k)
    vs.rotary(sh, plan, pos, None, k, None, alone, inverse=inverse)
    assert same_bits(alone, ko)
    vs.rotary(sh, plan, pos, q, None, qi, None, inverse=inverse)
    assert same_bits(qi, qo)


def test_rotary_of_more_tokens_than_a_launch_takes():
    sh, T, sections = vs.Shape.make(1, 1, 64, "f32"), 2 ** 24 + 5, (8, 12, 12)
    g = torch.Generator(device=DEV).manual_seed(3)
    k = torch.randn((T, 1, 64), generator=g, device=DEV)
    pos = torch.randint(-100000, 100000, (3, T), generator=g, device=DEV, dtype=torch.int32)
    out = torch.full_like(k, float("nan"))
    vs.rotary(sh, vs.RotaryPlan(64, sections), pos, None, k, None, out)
    some = [0, 1, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, 2 ** 24 - 1, 2 ** 24, T - 1]
    where = pos[:, some].cpu().numpy()
    want = ref.rotate(f64(k[some]), where, sections, 1e6, True)
    assert (np.abs(f64(out[some]) - want) <= rotary_bound(f64(k[some]), want, where, torch.float32)).all()
    assert torch.isfinite(out).all()


def test_rotary_inverse_is_the_gradient():
    """The rotation is linear: <rot(x), y> = <x, inv(y)> for all x, y, and its differences are itself.  fp32: each of the two
    sums of n products is off by at most sum|x||y| 2^-20.5 (the rotation, see rotary_bound) in any order of 64-bit sums."""
    sh, T = vs.Shape.make(4, 2, 64, "f32"), 50
    plan = vs.RotaryPlan(64, (8, 12, 12), 1e4)
    g = torch.Generator(device=DEV).manual_seed(3)
    x, y, d = (torch.randn((T, 4, 64), generator=g, device=DEV) for _ in range(3))
    pos = torch.randint(0, 5000, (3, T), generator=g, device=DEV, dtype=torch.int32)

    def rot(t, inverse=False):
        o = torch.empty_like(t)
        vs.rotary(sh, plan, pos, t, None, o, None, inverse=inverse)
        return o.double()

    reach = (x.double().norm() * y.double().norm()).item()
    assert abs(((rot(x) * y.double()).sum() - (x.double() * rot(y, True)).sum()).item()) <= 2 * 2.0 ** -20.5 * reach
    h = 2.0 ** -6
    slope = ((rot(x + h * d) - rot(x - h * d)) * y.double()).sum() / (2 * h)        # of <rot(x), y> along d
    grad = (rot(y, True) * d.double()).sum()
    # (x + h d is rounded to 2^-24 of itself, and each rotation is good to 2^-20.5: over 2 h)
    off = (2.0 ** -20.5 + 2.0 ** -24) * (x.double().norm() + h * d.double().norm()) * y.double().norm() * 2 / (2 * h) + 2.0 ** -20.5 * y.double().norm() * d.double().norm()
    assert abs(slope - grad).item() <= off.item()


# ---------------------------------------------------------------------------- rows written and read back
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("before,T,first", [(0, 1, 0), (0, 70, 0), (31, 1, 0), (31, 2, 0), (32, 32, 0), (5, 170, 169), (17, 64, 3), (63, 65, 0), (1, 31, 0)])
def test_rows_written_and_read_back(hq, hkv, before, T, first):
    sh, n, kept = vs.Shape.make(hq, hkv, 128, "bf16"), 3, T - first
    cap = before + kept + 3
    slab = slab_of(sh, n, cap)
    lens = lens_array([0] * n)
    pk, pv = rows(1, n, before, hkv, 128), rows(2, n, before, hkv, 128)
    if before:
        vs.cache8_append(sh, slab, cap, lens, pk, pv)
    k, v = rows(3, n, T, hkv, 128), rows(4, n, T, hkv, 128)
    k[0, first] = 0.0
    v[1, T - 1, 0, 7:] = 0.0
    k[2, T - 1] = torch.finfo(torch.bfloat16).tiny * 1.5   # all of it below the smallest scale's step: zeros or single steps
    v[2, first] = torch.finfo(torch.bfloat16).max
    was = slab.clone()
    vs.cache8_append(sh, slab, cap, lens, k, v, first_kept=first)
    assert list(lens) == [before + kept] * n
    ko, vo = (torch.empty((n, before + kept, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, slab, cap, lens, None, ko, vo)
    for got, old, new in ((ko, pk, k), (vo, pv, v)):
        assert torch.equal(got.cpu(), held(torch.cat([old, new[:, first:]], 1)))
    # row by row: the same bytes, those that belong to no row included
    one = slab_of(sh, n, cap)
    lens1 = lens_array([0] * n)
    every_k, every_v = torch.cat([pk, k[:, first:]], 1), torch.cat([pv, v[:, first:]], 1)
    for r in range(before + kept):
        vs.cache8_append(sh, one, cap, lens1, every_k[:, r:r + 1].contiguous(), every_v[:, r:r + 1].contiguous())
    assert same_bits(one, slab)
    # a row and head is 128 + 128 + 4 bytes; nothing else was touched
    assert (slab != was).sum().item() <= n * kept * hkv * 260
    # some of the rows
    some = min(3, before + kept)
    firsts = lens_array([before + kept - some, 0, (before + kept - some) // 2])
    k3, v3 = torch.empty((n, some, hkv, 128), dtype=torch.bfloat16, device=DEV), torch.empty((n, some, hkv, 128), dtype=torch.bfloat16, device=DEV)
    vs.cache8_read(sh, slab, cap, lens, firsts, k3, v3)
    for i in range(n):
        assert same_bits(k3[i], ko[i, firsts[i]:firsts[i] + some]) and same_bits(v3[i], vo[i, firsts[i]:firsts[i] + some])


@pytest.mark.parametrize("hq,hkv,T,first", [(28, 4, 1400, 0), (8, 8, 701, 1), (5, 5, 1111, 7)])
def test_many_rows_written_and_read_back(hq, hkv, T, first):
    """As many as go in blocks, behind rows that end anywhere in one, of which nothing else may change; the same bytes as written row by row."""
    sh, lens0, kept = vs.Shape.make(hq, hkv, 128, "bf16"), [5, 32, 63], T - first
    cap = 64 + T
    k, v = rows(120, 3, T, hkv, 128), rows(121, 3, T, hkv, 128)
    slab, lens = slab_of(sh, 3, cap, fill=0x5A), lens_array(lens0)
    one = slab.clone()
    vs.cache8_append(sh, slab, cap, lens, k, v, first_kept=first)
    assert list(lens) == [n + kept for n in lens0]
    for i, n0 in enumerate(lens0):
        part, n = one[i], lens_array([n0])
        for t in range(first, T, 300):
            e = min(t + 300, T)
            vs.cache8_append(sh, part, cap, n, k[i:i + 1, t:e].contiguous(), v[i:i + 1, t:e].contiguous())
    assert same_bits(slab, one)
    ko, vo = (torch.empty((3, kept, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, slab, cap, lens, lens_array(lens0), ko, vo)
    assert torch.equal(ko.cpu(), held(k[:, first:])) and torch.equal(vo.cpu(), held(v[:, first:]))
    kr, vr = (torch.empty((3, 9, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    at = 700 - first - 20
    vs.cache8_read(sh, slab, cap, lens, lens_array([n + at for n in lens0]), kr, vr)
    assert same_bits(kr, ko[:, at:at + 9]) and same_bits(vr, vo[:, at:at + 9])


def test_many_caches_of_different_lengths_and_a_longer_capacity():
    sh, n, T = vs.Shape.make(8, 2, 128, "bf16"), 131, 5
    before = [(7 * i) % 90 for i in range(n)]
    cap = 96
    slab = slab_of(sh, n, cap)
    k, v = rows(5, n, 90 + T, 2, 128), rows(6, n, 90 + T, 2, 128)
    lens = lens_array([0] * n)
    vs.cache8_append(sh, slab, cap, lens, k[:, :90].contiguous(), v[:, :90].contiguous())
    for i in range(n):
        lens[i] = before[i]                      # cut back, and grown again from there
    vs.cache8_append(sh, slab, cap, lens, k[:, 90:].contiguous(), v[:, 90:].contiguous())
    assert list(lens) == [b + T for b in before]
    ko, vo = (torch.empty((n, T, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, slab, cap, lens, lens_array(before), ko, vo)
    assert torch.equal(ko.cpu(), held(k[:, 90:])) and torch.equal(vo.cpu(), held(v[:, 90:]))
    # the bytes of the first rows, under another capacity
    i, m = 12, before[12] + T
    longer = slab_of(sh, 1, 700)
    size = vs.cache8_bytes(sh, m)
    longer[0, :size] = slab[i, :size]
    ka, va = (torch.empty((1, m, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, longer, 700, lens_array([m]), None, ka, va)
    want = torch.cat([k[i, :before[i]], k[i, 90:]])
    assert torch.equal(ka[0].cpu(), held(want))


def test_rows_that_are_not_finite():
    """Such a row stands for NaN in the head and tensor that it is in, and for nothing less anywhere else."""
    sh = vs.Shape.make(4, 2, 128, "bf16")
    k, v = rows(7, 1, 40, 2, 128), rows(8, 1, 40, 2, 128)
    k[0, 3, 1, 5], v[0, 33, 0, 127], v[0, 20, 1, 0] = float("inf"), float("nan"), float("-inf")
    slab, lens = slab_of(sh, 1, 64), lens_array([0])
    vs.cache8_append(sh, slab, 64, lens, k, v)
    ko, vo = (torch.empty((1, 40, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, slab, 64, lens, None, ko, vo)
    for got, x in ((ko, k), (vo, v)):
        bad = ~torch.isfinite(x.float()).all(-1)
        assert bad.any() and torch.isnan(got[bad].float()).all()
        clean = torch.where(bad[..., None], torch.zeros_like(x), x)
        assert torch.equal(got[~bad].cpu(), held(clean)[~bad.cpu()])
    # attention: the head that sees the row has no number to give, the other has
    q = rows(9, 1, 4, 128, loud=False)
    out, ws = torch.empty_like(q), vs.make_cache8_workspace(sh, 4, 64, 1, DEV)
    for n, expect in ((3, [False, False]), (4, [False, True]), (20, [False, True]), (40, [True, True])):
        vs.cache8_decode_attn(sh, slab, 64, lens_array([n]), q, None, None, out, ws)
        nan = torch.isnan(out.float()[0].view(2, 2 * 128)).all(-1).tolist()
        some = torch.isnan(out.float()[0].view(2, 2 * 128)).any(-1).tolist()
        assert nan == some == expect, n
    q[0, 2, 9] = float("nan")
    vs.cache8_decode_attn(sh, slab, 64, lens_array([3]), q, None, None, out, ws)
    assert torch.isnan(out.float()[0, 2]).all() and torch.isfinite(out.float()[0, [0, 1, 3]]).all()


# ---------------------------------------------------------------------------- decode
def decode_case(hq, hkv, lens0, seed, append=True, gain=1.0, cap=None, loud=True):
    sh, S = vs.Shape.make(hq, hkv, 128, "bf16"), len(lens0)
    cap = cap or max(lens0) + 2
    slab = slab_of(sh, S, cap)
    k, v = rows(seed, S, max(max(lens0), 1), hkv, 128, loud=loud), rows(seed + 1, S, max(max(lens0), 1), hkv, 128, loud=loud)
    lens = lens_array([0] * S)
    vs.cache8_append(sh, slab, cap, lens, k, v)
    for i in range(S):
        lens[i] = lens0[i]
    q = (rows(seed + 2, S, hq, 128, loud=False, sigma=1.0) * gain).to(torch.bfloat16)
    kn, vn = (rows(seed + 3, S, hkv, 128, loud=loud), rows(seed + 4, S, hkv, 128, loud=loud)) if append else (None, None)
    return sh, slab, cap, lens, k, v, q, kn, vn


def check_decode(sh, out, i, q, k, v, kn, vn, n0, what):
    kk, vv = (ref.stands_for(f64(a[i, :n0] if b is None else torch.cat([a[i, :n0], b[i:i + 1]]))) for a, b in ((k, kn), (v, vn)))
    scale = float(np.float32(sh.softmax_scale))
    want, absolute, most = ref.attend(f64(q[i:i + 1]), kk, vv, [len(kk)], scale)
    bound = ref.decode_bound(f64(q[i]), kk, vv, want[0], absolute[0], most[0], scale)
    err = np.abs(f64(out[i]) - want[0])
    assert np.isfinite(err).all() and (err <= bound).all(), f"{what}: {(err / bound).max():.2f} of what it may be off"
    # the bound is for the worst case; on the whole the two roundings to bf16 show, each of at most 2^-8 and 2^-8 / sqrt(3) on average,
    # the first averaged over the keys' terms: 2^-7 of the size of the terms is twice that
    assert err.mean() <= 2.0 ** -8 * absolute.mean() + 2.0 ** -8 * np.abs(want).mean(), what


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("lens0,append,gain", [([0], True, 1), ([1], False, 1), ([31, 32, 33], True, 1), ([31, 32, 33, 64], False, 8),
                                               ([700], True, 4), ([0, 3000, 5, 129, 640], True, 1), ([127, 128, 129], False, 1)])
def test_decode_over_rows_in_8_bits(hq, hkv, lens0, append, gain):
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(hq, hkv, lens0, 100 + len(lens0), append, gain)
    ws = vs.make_cache8_workspace(sh, 0, cap, len(lens0), DEV)
    was = slab.clone()
    out = torch.full_like(q, float("nan"))
    vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
    torch.cuda.synchronize()
    assert list(lens) == [n + append for n in lens0]
    for i, n0 in enumerate(lens0):
        check_decode(sh, out, i, q, k, v, kn, vn, n0, f"{hq}/{hkv} heads, stream {i} of {lens0}")
    if not append:
        assert same_bits(slab, was)
        return
    # the new row is what vs_cache8_append would have written, byte by byte
    lens2 = lens_array(lens0)
    vs.cache8_append(sh, was, cap, lens2, kn[:, None].contiguous(), vn[:, None].contiguous())
    assert same_bits(slab, was)


def test_decode_of_more_streams_than_a_launch_takes():
    lens0 = [(37 * i) % 200 for i in range(150)]
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(8, 2, lens0, 300)
    ws = vs.make_cache8_workspace(sh, 0, cap, 150, DEV)
    out = torch.full_like(q, float("nan"))
    vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
    for i in (0, 1, 63, 64, 100, 127, 128, 149):
        check_decode(sh, out, i, q, k, v, kn, vn, lens0[i], f"stream {i}")
    assert list(lens) == [n + 1 for n in lens0]


def test_decode_steps_grow_a_cache_and_repeat_their_bits():
    """70 steps across block ends; the same steps again from the start (len set back) give the same bits."""
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(28, 4, [25, 600], 400, cap=700)
    ws = vs.make_cache8_workspace(sh, 0, cap, 2, DEV)
    g = torch.Generator(device=DEV).manual_seed(9)
    steps = [tuple(torch.randn((2, h, 128), generator=g, device=DEV).to(torch.bfloat16) for h in (28, 4, 4)) for _ in range(70)]
    seen = []
    for turn in range(2):
        lens[0], lens[1] = 25, 600
        for t, (q, kn, vn) in enumerate(steps):
            out = torch.empty_like(q)
            vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
            if turn == 0:
                seen.append(out)
            else:
                assert same_bits(out, seen[t]), t
    k = torch.cat([k[:, :25], torch.stack([s[1] for s in steps], 1)], 1)
    v = torch.cat([v[:, :25], torch.stack([s[2] for s in steps], 1)], 1)
    for t in (0, 6, 7, 38, 39, 69):
        check_decode(sh, seen[t], 0, steps[t][0], k, v, None, None, 26 + t, f"step {t}")


def test_decode_peaked_and_flat_and_extreme():
    """One key that takes everything, equal keys, large and tiny values, a query of zeros."""
    sh = vs.Shape.make(8, 1, 128, "bf16")
    n, ws = 500, vs.make_cache8_workspace(sh, 0, 500, 1, DEV)
    base_k, base_v = rows(20, 1, n, 1, 128), rows(21, 1, n, 1, 128)
    q = rows(22, 1, 8, 128, loud=False, sigma=1.0)
    cases = {"flat": (torch.ones_like(base_k), base_v, q), "zero query": (base_k, base_v, torch.zeros_like(q)),
             "tiny": (base_k * 2.0 ** -100, base_v * 2.0 ** -100, q * 2.0 ** -20),
             "large values": (base_k, base_v * 2.0 ** 100, q), "large scores": (base_k * 2.0 ** 20, base_v, q),
             "large query": (base_k * 2.0 ** -90, base_v, q * 2.0 ** 90)}
    peak_k = base_k.clone()
    peak_k[0, 333, 0] = q[0, 5].float().mul(40).to(torch.bfloat16)
    cases["peaked"] = (peak_k, base_v, q)
    for name, (k, v, qq) in cases.items():
        slab, lens = slab_of(sh, 1, n), lens_array([0])
        vs.cache8_append(sh, slab, n, lens, k, v)
        out = torch.full_like(qq, float("nan"))
        vs.cache8_decode_attn(sh, slab, n, lens, qq, None, None, out, ws)
        check_decode(sh, out, 0, qq, k, v, None, None, n, name)


@pytest.mark.parametrize("fill", [0x00, 0xFF, 0x3C])
def test_decode_with_a_workspace_that_was_not_prepared(fill):
    """Arrival counters that hold anything: a stream's first share does the stream.  Then prepared again, and a workspace of other use."""
    lens0 = [3000, 20, 700]
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(28, 4, lens0, 600)
    ws = torch.full((vs.cache8_workspace_bytes(sh, 0, cap, 3),), fill, dtype=torch.uint8, device=DEV)
    was = slab.clone()
    for turn in range(3):
        if turn == 2:
            vs.workspace_init(sh, ws)
        slab.copy_(was)
        lens = lens_array(lens0)
        out = torch.full_like(q, float("nan"))
        vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
        for i, n0 in enumerate(lens0):
            check_decode(sh, out, i, q, k, v, kn, vn, n0, f"turn {turn}, stream {i}")
        expect = was.clone()
        vs.cache8_append(sh, expect, cap, lens_array(lens0), kn[:, None].contiguous(), vn[:, None].contiguous())
        assert same_bits(slab, expect)


def test_decode_of_one_long_and_many_short_streams():
    """Shares that a second launch adds (a stream of 64000 rows beside one of 1 row), and no new row."""
    lens0 = [64000, 1]
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(8, 2, lens0, 610, append=False)
    ws = vs.make_cache8_workspace(sh, 0, cap, 2, DEV)
    out = torch.full_like(q, float("nan"))
    vs.cache8_decode_attn(sh, slab, cap, lens, q, None, None, out, ws)
    for i, n0 in enumerate(lens0):
        check_decode(sh, out, i, q, k, v, kn, vn, n0, f"stream {i}")


# ---------------------------------------------------------------------------- prefill
@pytest.mark.parametrize("hq,hkv", [(28, 4), (8, 1), (5, 5)])
@pytest.mark.parametrize("L,T,kept", [(0, 1, 1), (0, 50, 50), (1, 1, 0), (31, 2, 2), (32, 170, 1), (33, 37, 37), (700, 37, 37), (711, 170, 1), (2000, 1, 1),
                                      (4424, 170, 1), (63, 300, 300)])
def test_prefill_over_rows_in_8_bits(hq, hkv, L, T, kept):
    s = AttnShape(hq, hkv, 128, "bf16")
    sh, cap = vs_shape(s), L + T
    slab, lens = slab_of(sh, 1, cap), lens_array([0])
    k, v = rows(30, 1, max(L, 1), hkv, 128, loud=False), rows(31, 1, max(L, 1), hkv, 128, loud=False)
    if L:
        vs.cache8_append(sh, slab, cap, lens, k, v)
    q, kt, vt = rows(32, T, hq, 128, loud=False, sigma=2.0), rows(33, T, hkv, 128, loud=False), rows(34, T, hkv, 128, loud=False)
    cache = vs.Cache8(slab[0], cap, L)
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)
    out = torch.full_like(q, float("nan"))
    was = slab.clone()
    vs.cache8_prefill_attn(sh, cache, q, kt, vt, out, ws, first_kept=T - kept)
    assert cache.len == L + kept
    kk, vv = (np.concatenate([ref.stands_for(f64(a[0, :L])), f64(b)]) if L else f64(b) for a, b in ((k, kt), (v, vt)))
    tokens = sorted({0, 1, T // 2, T - 2, T - 1} & set(range(T)))
    want, absolute, _ = ref.attend(f64(q)[tokens], kk, vv, [L + t + 1 for t in tokens], scale32(s))
    check_close(out[tokens], want, "bf16", f"L {L} T {T} heads {hq}/{hkv}", absolute=False, abs_v_out=absolute)
    assert torch.isfinite(out.float()).all()
    # the rows kept are what vs_cache8_append writes
    lens2 = lens_array([L])
    if kept:
        vs.cache8_append(sh, was, cap, lens2, kt[None], vt[None], first_kept=T - kept)
    assert same_bits(slab, was)


def test_prefill_keeps_what_is_not_finite_where_it_is_seen():
    """NaN and infinities in rows of the run: tokens before them do not see them, bit for bit; later ones get NaN where they come in."""
    s = AttnShape(8, 2, 128, "bf16")
    sh, L, T = vs_shape(s), 70, 75
    slab, lens = slab_of(sh, 1, L + T), lens_array([0])
    vs.cache8_append(sh, slab, L + T, lens, rows(80, 1, L, 2, 128), rows(81, 1, L, 2, 128))
    q, k, v = rows(82, T, 8, 128, loud=False), rows(83, T, 2, 128, loud=False), rows(84, T, 2, 128, loud=False)
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)

    def go(k, v):
        out = torch.full_like(q, float("nan"))
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, k, v, out, ws, first_kept=T)
        return out

    clean = go(k, v)
    assert torch.isfinite(clean.float()).all()
    for bad in ("nan", "inf", "-inf"):
        v2, k2 = v.clone(), k.clone()
        v2[20, 1, 77] = float(bad)
        out = go(k, v2)
        assert same_bits(out[:20], clean[:20]) and same_bits(out[:, :4], clean[:, :4])
        assert torch.isnan(out[20:, 4:, 77].float()).all()
        rest = [d for d in range(128) if d != 77]
        assert same_bits(out[20:, 4:][..., rest], clean[20:, 4:][..., rest])
        k2[64, 0, 3] = float(bad)
        out = go(k2, v)
        assert same_bits(out[:64], clean[:64]) and same_bits(out[:, 4:], clean[:, 4:])
        if bad == "nan":
            assert torch.isnan(out[64:, :4].float()).all()
    q2 = q.clone()
    q2[30, 5, 1] = float("inf")
    q, q2 = q2, q
    out = go(k, v)
    assert torch.isnan(out[30, 5].float()).all()
    out[30, 5] = clean[30, 5]
    assert same_bits(out, clean)


def test_prefill_extremes():
    """Large, tiny and zero queries and rows, one key that takes everything, rows of zeros that a query likes best."""
    s = AttnShape(8, 2, 128, "bf16")
    sh, L, T = vs_shape(s), 300, 40
    k, v, q = rows(90, 1, L, 2, 128), rows(91, 1, L, 2, 128), rows(92, T, 8, 128, loud=False, sigma=1.0)
    kt, vt = rows(93, T, 2, 128, loud=False), rows(94, T, 2, 128, loud=False)
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)
    zero_v = v.clone()
    zero_v[0, 7] = 0.0
    sink_k = k.clone()
    sink_k[0, 7, 0] = (q[3, 1].float() * 30).to(torch.bfloat16)
    cases = {"zero query": (k, v, q * 0, kt, vt), "tiny": (k * 2.0 ** -100, v * 2.0 ** -100, q * 2.0 ** -20, kt * 2.0 ** -100, vt * 2.0 ** -100),
             "large values": (k, v * 2.0 ** 100, q, kt, vt * 2.0 ** 100), "large query": (k * 2.0 ** -90, v, q * 2.0 ** 90, kt * 2.0 ** -90, vt),
             "sink": (sink_k, zero_v, q, kt, vt), "loud values that nobody looks at": (k, torch.where(torch.arange(L, device=DEV)[None, :, None, None] == 9, v * 2.0 ** 40, v),
                                                                                     q, kt, vt)}
    cases["loud values that nobody looks at"][0][0, 9] = (-q[:, :8:4].float().mean(0) * 400).to(torch.bfloat16)
    for name, (k1, v1, q1, kt1, vt1) in cases.items():
        slab, lens = slab_of(sh, 1, L + T), lens_array([0])
        vs.cache8_append(sh, slab, L + T, lens, k1, v1)
        out = torch.full_like(q1, float("nan"))
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q1, kt1, vt1, out, ws)
        kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k1, kt1), (v1, vt1)))
        scale = scale32(s)
        for t in (0, 3, 39):
            want, absolute, most = ref.attend(f64(q1[t:t + 1]), kk, vv, [L + t + 1], scale)
            bound = ref.decode_bound(f64(q1[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale)
            err = np.abs(f64(out[t]) - want[0])
            assert np.isfinite(err).all() and (err <= bound).all(), f"{name}, token {t}: {(err / bound).max():.2f}"


@pytest.mark.parametrize("L,T", [(900, 40), (900, 3)])
def test_prefill_of_values_near_the_smallest(L, T):
    """Values of 2^-114: what the splits of a row pass on is scaled up into fp16, and down again without loss."""
    s = AttnShape(8, 2, 128, "bf16")
    sh = vs_shape(s)
    slab, lens = slab_of(sh, 1, L + T), lens_array([0])
    k, kt, q = rows(95, 1, L, 2, 128), rows(96, T, 2, 128, loud=False), torch.zeros((T, 8, 128), dtype=torch.bfloat16, device=DEV)
    v, vt = torch.full_like(k, 2.0 ** -114), torch.full_like(kt, -(2.0 ** -114))
    vs.cache8_append(sh, slab, L + T, lens, k, v)
    out = torch.full_like(q, float("nan"))
    vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, kt, vt, out, vs.make_cache8_workspace(sh, T, L, 0, DEV))
    kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k, kt), (v, vt)))
    for t in (0, T - 1):
        want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale32(s))
        bound = ref.decode_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale32(s))
        assert (np.abs(f64(out[t]) - want[0]) <= bound).all(), t


@pytest.mark.parametrize("hq,hkv,L,T", [(8, 2, 300, 40), (8, 2, 1000, 3), (28, 4, 300, 400), (28, 4, 300, 1000), (28, 4, 9000, 170)])
def test_prefill_of_rows_of_very_different_sizes(hq, hkv, L, T):
    """V in rows of zeros that a query likes best, first or throughout, of sizes 2^-40 .. 2^40, very large or very small first rows."""
    s = AttnShape(hq, hkv, 128, "bf16")
    sh = vs_shape(s)
    k, v = rows(110, 1, L, hkv, 128), rows(111, 1, L, hkv, 128)
    q, kt, vt = rows(112, T, hq, 128, loud=False, sigma=1.0), rows(113, T, hkv, 128, loud=False), rows(114, T, hkv, 128, loud=False)
    like = (q.float().reshape(T, hkv, hq // hkv, 128).mean((0, 2)) * 300).to(torch.bfloat16)     # [Hkv][128]
    size = torch.exp2(torch.randint(-40, 41, (1, L, hkv, 1), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).float())
    row = torch.arange(L, device=DEV)[None, :, None, None]
    first = row < 40
    sink = torch.where(first, like[None, None], k)
    cases = {"first rows of zeros": (k, torch.where(first, 0.0, v)), "first rows of zeros liked best": (sink, torch.where(first, 0.0, v)),
             "all zeros": (k, v * 0), "many sizes": (k, v * size), "first rows large": (k, torch.where(first, v * 2.0 ** 100, v)),
             "first rows tiny": (k, torch.where(first, v * 2.0 ** -100, v)), "a tiny row liked best": (torch.where(row == 37, like[None, None], k), torch.where(row == 37, v * 2.0 ** -90, v)),
             "last rows large": (k, torch.where(row >= L - 20, v * 2.0 ** 60, v))}
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)
    for name, (k1, v1) in cases.items():
        k1, v1 = k1.to(torch.bfloat16), v1.to(torch.bfloat16)
        slab, lens = slab_of(sh, 1, L + T), lens_array([0])
        vs.cache8_append(sh, slab, L + T, lens, k1, v1)
        out = torch.full_like(q, float("nan"))
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, kt, vt, out, ws)
        kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k1, kt), (v1, vt)))
        for t in sorted({0, T // 2, T - 1}):
            want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale32(s))
            bound = ref.prefill_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale32(s))
            err = np.abs(f64(out[t]) - want[0])
            assert np.isfinite(err).all() and (err <= bound).all(), f"{name}, token {t}: {(err / bound).max():.2f}"


def test_prefill_of_the_longest_run():
    """4096 tokens over 50 rows, all kept: the rows kept fill planes of workgroups of their own."""
    s = AttnShape(8, 2, 128, "bf16")
    sh, L, T = vs_shape(s), 50, 4096
    slab, lens = slab_of(sh, 1, L + T), lens_array([0])
    k, v = rows(97, 1, L, 2, 128, loud=False), rows(98, 1, L, 2, 128, loud=False)
    vs.cache8_append(sh, slab, L + T, lens, k, v)
    q, kt, vt = rows(99, T, 8, 128, loud=False, sigma=2.0), rows(101, T, 2, 128, loud=False), rows(102, T, 2, 128, loud=False)
    was, out = slab.clone(), torch.full_like(q, float("nan"))
    cache = vs.Cache8(slab[0], L + T, L)
    vs.cache8_prefill_attn(sh, cache, q, kt, vt, out, vs.make_cache8_workspace(sh, T, L, 0, DEV), first_kept=0)
    assert cache.len == L + T
    kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k, kt), (v, vt)))
    tokens = [0, 31, 2047, 2048, 4095]
    want, absolute, _ = ref.attend(f64(q)[tokens], kk, vv, [L + t + 1 for t in tokens], scale32(s))
    check_close(out[tokens], want, "bf16", "longest run", absolute=False, abs_v_out=absolute)
    assert torch.isfinite(out.float()).all()
    vs.cache8_append(sh, was, L + T, lens, kt[None], vt[None])
    assert same_bits(slab, was)


# ---------------------------------------------------------------------------- as they are used together
def test_a_dialogue_in_8_bits():
    """Projection, positions, frames over the cache with their carriers kept, a question, a few answer tokens; then the cache cut back to
    before the question, and another question.  Every attention against the evaluation over what the cache stands for."""
    s = AttnShape(28, 4, 128, "bf16")
    sh, d, T, cap = vs_shape(s), 512, 50, 200
    g = torch.Generator(device=DEV).manual_seed(5)
    w = (torch.randn(((28 + 8) * 128, d), generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    plan = vs.RotaryPlan(128, (16, 24, 24))
    slab, lens = slab_of(sh, 1, cap), lens_array([0])
    cache = vs.Cache8(slab[0], cap, 0)
    ws = vs.make_cache8_workspace(sh, T, cap, 1, DEV)
    kk, vv = (np.zeros((0, 4, 128)) for _ in "kv")
    for f in range(40):
        e = torch.randn((T - 1, d), generator=g, device=DEV).to(torch.bfloat16)
        q, k, v = (torch.empty((T, h, 128), dtype=torch.bfloat16, device=DEV) for h in (28, 4, 4))
        vs.frame_qkv_project(sh, e, w, q, k, v)
        i = torch.arange(T, device=DEV)
        pos = torch.stack([1000 + f + 0 * i, i // 7, i % 7]).to(torch.int32)
        before = f64(k)
        vs.rotary(sh, plan, pos, q, k, q, k)
        turned = ref.rotate(before, pos.cpu().numpy(), (16, 24, 24), 1e6, True)
        assert (np.abs(f64(k) - turned) <= rotary_bound(before, turned, pos.cpu().numpy(), torch.bfloat16)).all()
        out = torch.empty_like(q)
        vs.cache8_prefill_attn(sh, cache, q, k, v, out, ws)
        if f in (0, 1, 31, 32, 33, 39):
            want, absolute, _ = ref.attend(f64(q), np.concatenate([kk, f64(k)]), np.concatenate([vv, f64(v)]), [f + t + 1 for t in range(T)], scale32(s))
            check_close(out, want, "bf16", f"frame {f}", absolute=False, abs_v_out=absolute)
        kk, vv = np.concatenate([kk, ref.stands_for(f64(k[-1:]))]), np.concatenate([vv, ref.stands_for(f64(v[-1:]))])
    assert cache.len == 40
    for n_q in (37, 5):
        cache.len = 40                      # (the second time: cut back to the frames)
        q, k, v = (rows(60 + n_q, n_q, h, 128, loud=False) for h in (28, 4, 4))
        out = torch.empty_like(q)
        vs.cache8_prefill_attn(sh, cache, q, k, v, out, ws, first_kept=0)
        lens = lens_array([cache.len])
        ka, va = np.concatenate([kk, ref.stands_for(f64(k))]), np.concatenate([vv, ref.stands_for(f64(v))])
        for step in range(6):
            q, k, v = (rows(70 + 10 * n_q + step, 1, h, 128, loud=False) for h in (28, 4, 4))
            out = torch.empty_like(q)
            vs.cache8_decode_attn(sh, slab, cap, lens, q, k, v, out, ws)
            ka, va = np.concatenate([ka, ref.stands_for(f64(k))]), np.concatenate([va, ref.stands_for(f64(v))])
            want, absolute, most = ref.attend(f64(q), ka, va, [len(ka)], scale32(s))
            assert (np.abs(f64(out) - want) <= ref.decode_bound(f64(q[0]), ka, va, want[0], absolute[0], most[0], scale32(s))).all(), step
        assert lens[0] == 40 + n_q + 6


def test_on_another_stream_and_captured():
    """Calls on a stream of their own, then captured into one graph and replayed among eager work: the same bits every time."""
    s = AttnShape(28, 4, 128, "bf16")
    sh, cap = vs_shape(s), 3000
    _, slab, _, _, k, v, q, kn, vn = decode_case(28, 4, [700, 2500], 500, cap=cap)
    T = 64
    qf, kf, vf = rows(501, T, 28, 128, loud=False), rows(502, T, 4, 128, loud=False), rows(503, T, 4, 128, loud=False)
    plan = vs.RotaryPlan(128, (16, 24, 24))
    pos = torch.arange(3 * T, device=DEV, dtype=torch.int32).view(3, T)
    ws = vs.make_cache8_workspace(sh, T, cap, 2, DEV)
    qr, kr, of, od = torch.empty_like(qf), torch.empty_like(kf), torch.empty_like(qf), torch.empty_like(q)
    back = [torch.empty((2, 40, 4, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    start = slab.clone()

    def pass_():
        lens = lens_array([700, 2500])
        cache = vs.Cache8(slab[1], cap, 2500)
        vs.rotary(sh, plan, pos, qf, kf, qr, kr)
        vs.cache8_prefill_attn(sh, cache, qr, kr, vf, of, ws, first_kept=T - 30)
        lens[1] = cache.len
        vs.cache8_append(sh, slab[0:1], cap, (ctypes.c_int32 * 1).from_buffer(lens), kr[None], vf[None], first_kept=T - 9)
        vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, od, ws)
        vs.cache8_read(sh, slab, cap, lens, lens_array([lens[0] - 40, lens[1] - 40]), *back)
        return list(lens)

    assert pass_() == [710, 2531]
    torch.cuda.synchronize()
    outs = (slab, qr, kr, of, od, *back)
    first = [t.clone() for t in outs]

    def again(run):
        for t in outs[1:]:
            t.fill_(float("nan"))
        slab.copy_(start)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        for t, want in zip(outs, first):
            assert same_bits(t, want)

    side = torch.cuda.Stream()

    def aside():
        with torch.cuda.stream(side):
            pass_()
    again(aside)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pass_()
    for turn in range(3):
        again(graph.replay)
        again(pass_)


def test_two_graphs_over_one_workspace():
    """A prefill and a decoding step in a graph each, replayed in turn with eager calls between, all over the same workspace."""
    sh, slab, cap, _, k, v, q, kn, vn = decode_case(28, 4, [2500, 900], 700, cap=2600)
    T = 37
    qf, kf, vf = rows(701, T, 28, 128, loud=False), rows(702, T, 4, 128, loud=False), rows(703, T, 4, 128, loud=False)
    ws = vs.make_cache8_workspace(sh, T, cap, 2, DEV)
    of, od = torch.empty_like(qf), torch.empty_like(q)

    def frame():
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[1], cap, 900), qf, kf, vf, of, ws, first_kept=T)

    def step():
        vs.cache8_decode_attn(sh, slab, cap, lens_array([2500, 900]), q, kn, vn, od, ws)

    frame(), step()
    torch.cuda.synchronize()
    want = of.clone(), od.clone()
    graphs = []
    for call in (frame, step):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for order in ((0, 1), (1, 0), (1, 1), (0, 0), (0, 1)):
        of.fill_(float("nan")), od.fill_(float("nan"))
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i, (got, first) in enumerate(zip((of, od), want)):
            assert i not in order or same_bits(got, first)
        step(), frame()
        torch.cuda.synchronize()
        assert same_bits(of, want[0]) and same_bits(od, want[1])


def test_more_than_4_gib_of_rows():
    """A cache whose bytes pass 2^32, and a second one behind it: rows that were never written hold whole numbers and scales of 0
    there (the memory is cleared), K of zeros and V of -128 * 0."""
    sh = vs.Shape.make(8, 8, 128, "bf16")
    far = 2_200_000
    cap = far + 100
    slab = torch.zeros((2, vs.cache8_bytes(sh, cap)), dtype=torch.uint8, device=DEV)
    assert slab.shape[1] > 2 ** 32
    k, v = rows(40, 2, 40, 8, 128, loud=False), rows(41, 2, 40, 8, 128, loud=False, sigma=2.0)
    lens = lens_array([far, far])
    vs.cache8_append(sh, slab, cap, lens, k, v)
    ko, vo = (torch.empty((2, 40, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    vs.cache8_read(sh, slab, cap, lens, lens_array([far, far]), ko, vo)
    assert torch.equal(ko.cpu(), held(k)) and torch.equal(vo.cpu(), held(v))
    q = (k.float()[:, 7] * 60).to(torch.bfloat16)          # the key at `far` + 7 stands out among 2.2 million of score 0
    kn, vn = rows(42, 2, 8, 128, loud=False), rows(43, 2, 8, 128, loud=False)
    out, ws = torch.empty_like(q), vs.make_cache8_workspace(sh, 0, cap, 2, DEV)
    vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
    assert list(lens) == [far + 41] * 2
    scale = float(np.float32(sh.softmax_scale))
    for i in range(2):
        kk, vv = (ref.stands_for(f64(torch.cat([a[i], b[i:i + 1]]))) for a, b in ((k, kn), (v, vn)))
        for h in range(8):
            z = kk[:, h] @ f64(q[i, h]) * scale
            w = np.exp(z - z.max())
            total = w.sum() + far * np.exp(-z.max())
            want, absolute = w @ vv[:, h] / total, w @ np.abs(vv[:, h]) / total
            # (as decode_bound, the sums over the few rows that are not zero; 70000 blocks' worth of zeros add nothing but to the denominator,
            # whose fp32 sum of equal terms over a wavefront's share is off by at most 2^-24 a term)
            e = 2.0 ** -15 * np.abs(f64(q[i, h])).max() * np.abs(kk[:, h]).sum(-1).max() * scale + 2.0 ** -21 * np.abs(z).max()
            terms = far / 64                                # of one lane, if a single wavefront took an eighth of the rows
            bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + np.expm1(2 * e) + terms * 2.0 ** -24) * 1.01 * absolute + 2.0 ** -15 * absolute.max()
            assert (np.abs(f64(out[i, h]) - want) <= bound).all(), (i, h)


# ---------------------------------------------------------------------------- the ends of the range
@pytest.mark.parametrize("q_up,k_up,scale_up", [(-112, 112, 0), (-109, 109, 0), (-122, 118, 0), (-60, 118, -57), (-20, 118, -97), (112, -112, 0), (60, -90, 28)])
def test_small_queries_over_large_keys_and_the_reverse(q_up, k_up, scale_up):
    """Q, K and the softmax scale times powers of two: the scores stay of ordinary size, and so does what a score may be off (see
    decode_bound).  Tokens over cached rows, over their own rows, and a step."""
    sh = vs.Shape.make(8, 2, 128, "bf16", 128 ** -0.5 * 2.0 ** scale_up)
    scale, L, T = float(np.float32(sh.softmax_scale)), 300, 40
    k, v = rows(130, 1, L, 2, 128, loud=False) * 2.0 ** k_up, rows(131, 1, L, 2, 128)
    q, kt, vt = rows(132, T, 8, 128, loud=False, sigma=2.0) * 2.0 ** q_up, rows(133, T, 2, 128, loud=False) * 2.0 ** k_up, rows(134, T, 2, 128)
    slab, lens = slab_of(sh, 1, L + T), lens_array([0])
    vs.cache8_append(sh, slab, L + T, lens, k, v)
    ws = vs.make_cache8_workspace(sh, T, L + T, 1, DEV)
    out = torch.full_like(q, float("nan"))
    vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, kt, vt, out, ws, first_kept=T)
    kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k, kt), (v, vt)))
    for t in (0, 3, 39):
        want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale)
        bound = ref.prefill_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale)
        err = np.abs(f64(out[t]) - want[0])
        assert np.isfinite(err).all() and (err <= bound).all(), f"token {t}: {(err / bound).max():.2f}"
    step = torch.full_like(q[:1], float("nan"))
    vs.cache8_decode_attn(sh, slab, L + T, lens, q[:1], kt[:1], vt[:1], step, ws)
    check_decode(sh, step, 0, q[:1], k, v, kt[:1], vt[:1], L, "step")


@pytest.mark.parametrize("hq,hkv,L,T", [(8, 2, 300, 40), (8, 2, 1000, 3), (28, 4, 300, 400), (28, 4, 9000, 170)])
def test_prefill_where_one_side_is_far_larger(hq, hkv, L, T):
    """V of the run and of the cache, and of a cache's first and last rows, tens of powers of two apart, either way round; up to the largest bf16."""
    s = AttnShape(hq, hkv, 128, "bf16")
    sh = vs_shape(s)
    k, v = rows(140, 1, L, hkv, 128), rows(141, 1, L, hkv, 128, loud=False)
    q, kt, vt = rows(142, T, hq, 128, loud=False, sigma=1.0), rows(143, T, hkv, 128, loud=False), rows(144, T, hkv, 128, loud=False)
    row = torch.arange(L, device=DEV)[None, :, None, None]
    late, one = row >= L // 2 + 5, row == L - 7
    top = torch.full_like(vt, torch.finfo(torch.bfloat16).max)
    top[:, :, ::2] *= -1
    zeros = torch.where(row < 200, 0.0, v)
    cases = {"own rows large": (v, vt * 2.0 ** 112), "own rows largest": (v, top), "all rows largest": (v * 0 + top[0, 0], top),
             "own rows 2^140 up": (v * 2.0 ** -55, vt * 2.0 ** 85), "own rows 2^200 up": (v * 2.0 ** -100, vt * 2.0 ** 100),
             "cached rows 2^200 up": (v * 2.0 ** 100, vt * 2.0 ** -100), "both large": (v * 2.0 ** 122, vt * 2.0 ** 122),
             "own rows 2^60 up, both large": (v * 2.0 ** 62, vt * 2.0 ** 122), "last rows 2^180 up": (torch.where(late, v * 2.0 ** 100, v * 2.0 ** -80), vt),
             "last rows 2^205 up": (torch.where(late, v * 2.0 ** 122, v * 2.0 ** -83), vt), "last rows 2^120 up": (torch.where(late, v * 2.0 ** 40, v * 2.0 ** -80), vt * 2.0 ** 40),
             "one row 2^200 up": (torch.where(one, v * 2.0 ** 120, v * 2.0 ** -80), vt * 2.0 ** -80), "first rows zeros, last large": (torch.where(late, zeros * 2.0 ** 110, zeros), vt),
             "first rows zeros, the others tiny": (zeros * 2.0 ** -105, vt * 2.0 ** -105), "last rows large, own larger": (torch.where(late, v * 2.0 ** 100, v), vt * 2.0 ** 120)}
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)
    wrong = []
    for name, (v1, vt1) in cases.items():
        v1, vt1 = v1.to(torch.bfloat16), vt1.to(torch.bfloat16)
        slab, lens = slab_of(sh, 1, L + T), lens_array([0])
        vs.cache8_append(sh, slab, L + T, lens, k, v1)
        out = torch.full_like(q, float("nan"))
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, kt, vt1, out, ws)
        kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k, kt), (v1, vt1)))
        for t in sorted({0, T // 2, T - 1}):
            want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale32(s))
            bound = ref.prefill_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale32(s))
            err = off_by(out[t], want[0])
            if not (err <= bound).all():
                wrong.append(f"{name}, token {t}: {(err / bound).max():.2f}")
    assert not wrong, wrong


@pytest.mark.parametrize("hq,hkv,L,T", [(8, 2, 300, 40), (28, 4, 9000, 170)])
def test_prefill_with_large_rows_that_nobody_looks_at(hq, hkv, L, T):
    """A cached row of 2^80, or an own one of 2^110, whose score is some 400 under the others': what is seen is 2^-40 and keeps its bits."""
    s = AttnShape(hq, hkv, 128, "bf16")
    sh = vs_shape(s)
    g = torch.Generator(device=DEV).manual_seed(7)
    k, v = rows(150, 1, L, hkv, 128, loud=False), rows(151, 1, L, hkv, 128, loud=False) * 2.0 ** -40
    q, kt, vt = rows(152, T, hq, 128, loud=False, sigma=0.2), rows(153, T, hkv, 128, loud=False), rows(154, T, hkv, 128, loud=False) * 2.0 ** -40
    q[..., 0] = 30.0
    k[..., 0], kt[..., 0] = 0.0, 0.0
    cached, own, own_large = (torch.randint(0, n, (2,), generator=g, device=DEV) for n in (L, T, T))
    k2, v2, kt2, vt2 = k.clone(), v.clone(), kt.clone(), vt.clone()
    k2[0, cached, :, 0] = -150.0                      # a score of -150 * 30 / sqrt(128) = -398
    v2[0, cached] *= 2.0 ** 120
    kt2[own_large, :, 0] = -150.0
    vt2[own_large] = vt2[own_large] * 2.0 ** 75 * 2.0 ** 75
    ws = vs.make_cache8_workspace(sh, T, L, 0, DEV)
    for name, (k1, v1, kt1, vt1) in {"cached": (k2, v2, kt, vt), "own": (k, v, kt2, vt2), "both": (k2, v2, kt2, vt2)}.items():
        slab, lens = slab_of(sh, 1, L + T), lens_array([0])
        vs.cache8_append(sh, slab, L + T, lens, k1, v1)
        out = torch.full_like(q, float("nan"))
        vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L + T, L), q, kt1, vt1, out, ws, first_kept=T)
        kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k1, kt1), (v1, vt1)))
        for t in (0, T // 2, T - 1):
            want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale32(s))
            # (a key whose probability is under 2^-500 adds nothing, whatever became of it: the bounds without its value)
            seen = np.abs(kk[:L + t + 1, 0, 0]) < 100
            bound = ref.prefill_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1] * seen[:, None, None], want[0], absolute[0], most[0], scale32(s))
            err = off_by(out[t], want[0])
            assert (err <= bound).all(), f"{name}, token {t}: {(err / bound).max():.2f}"


@pytest.mark.parametrize("hq,hkv", [(8, 1), (28, 4)])
@pytest.mark.parametrize("lens0", [[1, 40], [500, 3], [3000, 33, 700], [64000, 1]])
def test_decode_of_values_up_to_the_largest(hq, hkv, lens0):
    """Long flat keys over V near the largest bf16, throughout, in some rows, in the new row alone: a mean is no larger than what it is of."""
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(hq, hkv, lens0, 160, loud=False)
    ws = vs.make_cache8_workspace(sh, 0, cap, len(lens0), DEV)
    row = torch.arange(k.shape[1], device=DEV)[None, :, None, None]
    largest = torch.full_like(v, torch.finfo(torch.bfloat16).max)
    rising = (k.float() + q.float()[:, None, ::hq // hkv] * row / k.shape[1] * 0.5).to(torch.bfloat16)
    cases = {"flat, largest": (torch.ones_like(k), largest, torch.ones_like(kn), largest[:, 0].contiguous()), "flat, 2^118": (torch.ones_like(k), v * 2.0 ** 118, kn, vn * 2.0 ** 118),
             "2^122": (k, v * 2.0 ** 122, kn, vn * 2.0 ** 122), "rising scores, 2^122": (rising, v * 2.0 ** 122, kn, vn * 2.0 ** 122),
             "new row alone": (k, v, kn, vn * 2.0 ** 122), "every other block": (k, torch.where(row // 32 % 2 == 1, v * 2.0 ** 120, v), kn, vn),
             "last rows": (k, torch.where(row >= k.shape[1] // 2, v * 2.0 ** 120, v), kn, vn), "first rows": (k, torch.where(row < 70, v * 2.0 ** 120, v), kn, vn)}
    wrong = []
    for name, (k1, v1, kn1, vn1) in cases.items():
        if lens0[0] > 10000 and name not in ("flat, largest", "2^122", "last rows"):
            continue
        k1, v1, kn1, vn1 = (t.to(torch.bfloat16) for t in (k1, v1, kn1, vn1))
        lens = lens_array([0] * len(lens0))
        vs.cache8_append(sh, slab, cap, lens, k1, v1)
        for i, n in enumerate(lens0):
            lens[i] = n
        out = torch.full_like(q, float("nan"))
        vs.cache8_decode_attn(sh, slab, cap, lens, q, kn1, vn1, out, ws)
        scale = float(np.float32(sh.softmax_scale))
        for i, n0 in enumerate(lens0):
            kk, vv = (ref.stands_for(f64(torch.cat([a[i, :n0], b[i:i + 1]]))) for a, b in ((k1, kn1), (v1, vn1)))
            want, absolute, most = ref.attend(f64(q[i:i + 1]), kk, vv, [n0 + 1], scale)
            bound = ref.decode_bound(f64(q[i]), kk, vv, want[0], absolute[0], most[0], scale)
            err = off_by(out[i], want[0])
            if not (err <= bound).all():
                wrong.append(f"{name}, stream {i}: {(err / bound).max():.2f}")
    assert not wrong, wrong


def test_decode_with_large_rows_that_nobody_looks_at():
    """A row of 2^120 whose score is some 400 under the others', in one stream of two: what is seen is of ordinary size and keeps its bits."""
    lens0 = [700, 90]
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(28, 4, lens0, 170, loud=False)
    ws = vs.make_cache8_workspace(sh, 0, cap, 2, DEV)
    q[..., 0] = 30.0
    k[..., 0], kn[..., 0] = 0.0, 0.0
    k[:, [5, 69], :, 0] = -150.0                     # a score of -150 * 30 / sqrt(128) = -398
    clean = v.clone()
    v[:, [5, 69]] *= 2.0 ** 120
    clean[:, [5, 69]] = 0.0
    lens = lens_array([0, 0])
    vs.cache8_append(sh, slab, cap, lens, k, v)
    lens[0], lens[1] = lens0
    out = torch.full_like(q, float("nan"))
    vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
    for i, n0 in enumerate(lens0):
        check_decode(sh, out, i, q, k, clean, kn, vn, n0, f"stream {i}")


@pytest.mark.parametrize("hq,hkv,lens0", [
    (28, 4, [(131 * i) % 1500 for i in range(64)]),                      # a workgroup for every stream and KV head, nothing shared out
    (28, 4, [(131 * i) % 1500 for i in range(70)]),                      # and a second launch of few streams, shared out
    (16, 4, [200 + 37 * i for i in range(39)] + [6000]),                 # shares of a size that is searched for
    (8, 8, [5500] + [(91 * i) % 300 for i in range(31)]),                # a long one among short ones, nothing shared out
    (8, 2, [(211 * i) % 900 for i in range(63)] + [2500] + [3000, 40])])  # two launches that are both shared out, over the same counters
def test_decode_of_many_streams(hq, hkv, lens0):
    S = len(lens0)
    sh, slab, cap, lens, k, v, q, kn, vn = decode_case(hq, hkv, lens0, 180)
    ws = vs.make_cache8_workspace(sh, 0, cap, S, DEV)
    was, expect = slab.clone(), slab.clone()
    first = None
    for turn in range(2):
        slab.copy_(was)
        lens, out = lens_array(lens0), torch.full_like(q, float("nan"))
        vs.cache8_decode_attn(sh, slab, cap, lens, q, kn, vn, out, ws)
        assert list(lens) == [n + 1 for n in lens0]
        first = out if first is None else first
    assert same_bits(first, out)
    for i in sorted({0, 1, 2, S // 2, 62, 63, 64, 65, S - 3, S - 2, S - 1} & set(range(S))):
        check_decode(sh, out, i, q, k, v, kn, vn, lens0[i], f"stream {i}")
    assert torch.isfinite(out.float()).all()
    vs.cache8_append(sh, expect, cap, lens_array(lens0), kn[:, None].contiguous(), vn[:, None].contiguous())
    assert same_bits(slab, expect)


@pytest.mark.parametrize("at", [3, 4090, 4104, 5000, 8999])
def test_prefill_finds_a_large_row_anywhere_in_a_long_share(at):
    """One row of 2^100 among 9000 of 2^-80 that nothing splits: every wavefront walks 70 blocks."""
    s = AttnShape(28, 4, 128, "bf16")
    sh, L, T = vs_shape(s), 9000, 600
    k, v = rows(190, 1, L, 4, 128, loud=False), rows(191, 1, L, 4, 128, loud=False) * 2.0 ** -80
    v[0, at] *= 2.0 ** 120
    v[0, at] *= 2.0 ** 60
    q, kt, vt = rows(192, T, 28, 128, loud=False, sigma=1.0), rows(193, T, 4, 128, loud=False), rows(194, T, 4, 128, loud=False) * 2.0 ** -80
    slab, lens = slab_of(sh, 1, L), lens_array([0])
    vs.cache8_append(sh, slab, L, lens, k, v)
    out = torch.full_like(q, float("nan"))
    vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], L, L), q, kt, vt, out, vs.make_cache8_workspace(sh, T, L, 0, DEV), first_kept=T)
    kk, vv = (np.concatenate([ref.stands_for(f64(a[0])), f64(b)]) for a, b in ((k, kt), (v, vt)))
    for t in (0, T - 1):
        want, absolute, most = ref.attend(f64(q[t:t + 1]), kk, vv, [L + t + 1], scale32(s))
        bound = ref.prefill_bound(f64(q[t]), kk[:L + t + 1], vv[:L + t + 1], want[0], absolute[0], most[0], scale32(s))
        err = off_by(out[t], want[0])
        assert (err <= bound).all(), f"token {t}: {(err / bound).max():.2f}"


def test_the_first_tokens_of_larger_buffers():
    """Tensors that go on behind the run's tokens: the same bits in front, nothing written behind.  Lengths through a pointer, as through an array."""
    sh, T, L, cap = vs.Shape.make(8, 2, 128, "bf16"), 11, 100, 130
    q, k, v = rows(200, 20, 8, 128, loud=False), rows(201, 20, 2, 128, loud=False), rows(202, 20, 2, 128, loud=False)
    pos = torch.arange(3 * T, device=DEV, dtype=torch.int32).view(3, T)
    plan, slab, lens = vs.RotaryPlan(128, (16, 24, 24)), slab_of(sh, 1, cap), lens_array([0])
    vs.cache8_append(sh, slab, cap, ctypes.cast(lens, ctypes.POINTER(ctypes.c_int32)), rows(203, 1, L, 2, 128), rows(204, 1, L, 2, 128))
    assert lens[0] == L
    ws = vs.make_cache8_workspace(sh, T, cap, 1, DEV)
    qo, ko, out, step = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    exact = [torch.empty_like(t[:T]) for t in (q, k, q)] + [torch.empty_like(q[:1])]
    vs.rotary(sh, plan, pos, q, k, qo, ko)
    vs.rotary(sh, plan, pos, q[:T], k[:T], exact[0], exact[1])
    vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], cap, L), q[:T], k, v, out, ws, first_kept=T)
    vs.cache8_prefill_attn(sh, vs.Cache8(slab[0], cap, L), q[:T], k[:T], v[:T], exact[2], ws, first_kept=T)
    vs.cache8_decode_attn(sh, slab, cap, lens_array([L]), q[:1], k, v, step, ws)
    vs.cache8_decode_attn(sh, slab, cap, lens_array([L]), q[:1], k[:1], v[:1], exact[3], ws)
    for got, want, n in zip((qo, ko, out, step), exact, (T, T, T, 1)):
        assert same_bits(got[:n], want) and (got[n:] == 7.0).all()
