"""Rotary positions and rows in 8 bits without a GPU: the plain evaluations themselves, and what the library refuses before it launches
anything."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

import operators_ref as ref
import paper_2503_09387_amd as vs
from paper_2503_09387_amd import binding

FAKE = 0x7F0000001000  # 16-byte aligned, never dereferenced: every call below must fail first
ODD = FAKE + 4


def _shape(hq=28, hkv=4, d=128, dt=vs.VS_BF16, scale=None):
    return vs.Shape.make(hq, hkv, d, dt, scale)


def _bf16(x):
    """Rounded to 8 significant bits."""
    m, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


# ---------------------------------------------------------------------------- the evaluations
def test_quantised_rows_in_exact_fractions():
    r = np.random.default_rng(0)
    x = _bf16(r.standard_normal((40, 128)) * 2.0 ** r.integers(-30, 30, (40, 1)))
    x[0] = 0.0
    x[1, 5:] = 0.0
    x[2] = _bf16(127.0 * 2.0 ** -7)
    x[3, 0], x[3, 1:] = 254.0, 1.0      # s = 2: ties everywhere
    q, s = ref.quantise(x)
    for i in range(40):
        most = max(abs(Fraction(v)) for v in x[i])
        scale = Fraction(float(s[i, 0]))
        if most:
            assert scale * 127 >= most and scale * 127 * Fraction(255, 256) <= most * Fraction(256, 255)
        bits = scale.numerator.bit_length() - (scale.numerator & -scale.numerator).bit_length() + 1
        assert bits <= 8
        for v, w in zip(x[i], q[i]):
            off = abs(Fraction(float(v)) / scale - int(w))
            assert off < Fraction(1, 2) or (off == Fraction(1, 2) and int(w) % 2 == 0)
        assert np.abs(q[i]).max() <= 127
    assert (q[0] == 0).all() and s[0, 0] == 2.0 ** -126
    assert s[3, 0] == 2.0 and q[3, 0] == 127 and (q[3, 1:] == 0).all()


def test_fp32_quotients_round_to_the_same_whole_numbers():
    """For every pair of 8-bit numbers that a row can hold beside its scale: the quotient in fp32, rounded, is the exact one's."""
    a = np.arange(128, 256, dtype=np.float64)          # significands of x
    for b in range(128, 256):                           # and of the scale
        for shift in range(-9, 9):
            x, s = np.ldexp(a, shift), float(b)
            ok = x / s <= 127.0
            exact = np.rint(x[ok] / s)                  # (a quotient of 8-bit numbers in fp64: far closer than 2^-17 of itself)
            assert np.array_equal(np.rint(x[ok].astype(np.float32) / np.float32(s)), exact)


def test_rotation_in_closed_form():
    x = np.zeros((4, 1, 64))
    x[:, 0, 0], x[:, 0, 31] = 1.0, 2.0
    pos = np.array([[0, 1, 2, -3], [5, 6, 7, 8], [9, 1, 4, 2]])
    y = ref.rotate(x, pos, (8, 12, 12), 100.0, True)
    assert np.allclose(y[:, 0, 0], np.cos(pos[0])) and np.allclose(y[:, 0, 32], np.sin(pos[0]))
    last = pos[2] * 100.0 ** (-31 / 32)
    assert np.allclose(y[:, 0, 31], 2 * np.cos(last)) and np.allclose(y[:, 0, 63], 2 * np.sin(last))
    y = ref.rotate(x, pos, (8, 12, 12), 100.0, False)
    assert np.allclose(y[:, 0, 0], np.cos(pos[0])) and np.allclose(y[:, 0, 1], np.sin(pos[0]))
    fifteenth = pos[1] * 100.0 ** (-15 / 32)
    assert np.allclose(y[:, 0, 30], -2 * np.sin(fifteenth)) and np.allclose(y[:, 0, 31], 2 * np.cos(fifteenth))
    z = np.random.default_rng(1).standard_normal((4, 3, 64))
    back = ref.rotate(ref.rotate(z, pos, (8, 4, 4), 1e4, True), pos, (8, 4, 4), 1e4, True, inverse=True)
    assert np.allclose(back, z) and np.array_equal(ref.rotate(z, pos, (8, 4, 4), 1e4, True)[..., 32:], z[..., 32:])


def test_attention_weights_of_the_evaluation():
    r = np.random.default_rng(2)
    q, k, v = r.standard_normal((2, 4, 8)), r.standard_normal((5, 2, 8)), r.standard_normal((5, 2, 8))
    out, absolute, most = ref.attend(q, k, v, [3, 5], 0.5)
    w = np.exp([q[0, 3] @ k[i, 1] * 0.5 for i in range(3)])
    assert np.allclose(out[0, 3], (w[:, None] * v[:3, 1]).sum(0) / w.sum())
    assert (absolute >= np.abs(out) - 1e-12).all() and (most >= absolute - 1e-12).all()


# ---------------------------------------------------------------------------- refusals
def test_rotary_argument_errors():
    L = vs.lib()
    plan = binding._CRotaryPlan()

    def make(d=128, sec=(16, 24, 24), theta=1e6, pairing=0, out=plan):
        return L.vs_rotary_plan_make(d, (ctypes.c_int32 * 3)(*sec), theta, pairing, ctypes.byref(out))

    assert L.vs_rotary_plan_make(128, None, 1e6, 0, ctypes.byref(plan)) == 1
    assert L.vs_rotary_plan_make(128, (ctypes.c_int32 * 3)(64, 0, 0), 1e6, 0, None) == 1
    assert make(d=96) == 3
    for sec in ((16, 24, 25), (0, 0, 0), (64, 8, 0), (-8, 40, 32), (4, 0, 0), (2 ** 31 - 1, 2 ** 31 - 1, 2)):
        assert make(sec=sec) == 2, sec
    assert make(theta=0.0) == 2 and make(theta=float("nan")) == 2 and make(theta=float("inf")) == 2 and make(pairing=2) == 2
    assert plan.head_dim == 0                                        # nothing was written
    assert make() == 0 and plan.head_dim == 128 and abs(plan.turns[0] * 2 * np.pi - 1.0) < 1e-15
    assert abs(plan.turns[63] * 2 * np.pi / 1e6 ** (-63 / 64) - 1) < 1e-14

    def rot(pos=FAKE, n=4, q=FAKE, k=FAKE, qo=FAKE, ko=FAKE, shape=_shape(), plan=plan):
        return L.vs_rotary(ctypes.byref(shape), ctypes.byref(plan), pos, n, q, k, 0, qo, ko, None)

    assert L.vs_rotary(None, ctypes.byref(plan), FAKE, 4, FAKE, FAKE, 0, FAKE, FAKE, None) == 1
    assert L.vs_rotary(ctypes.byref(_shape()), None, FAKE, 4, FAKE, FAKE, 0, FAKE, FAKE, None) == 1
    assert rot(pos=None) == 1 and rot(q=None, qo=None, k=None, ko=None) == 1
    assert rot(q=None) == 1 and rot(ko=None) == 1                    # an input without its output, and the reverse
    assert rot(n=0) == 2 and rot(n=2 ** 26 + 1) == 2
    assert rot(shape=_shape(4, 1, 64, vs.VS_F32)) == 2               # another head size than the plan's
    assert rot(shape=_shape(d=96)) == 3 and rot(shape=_shape(hq=28, hkv=5)) == 2
    assert rot(q=ODD) == 6 and rot(ko=ODD) == 6 and rot(pos=FAKE + 2) == 6
    assert rot(qo=FAKE + 256) == 2 and rot(ko=FAKE - 16) == 2        # overlaps its input without being it
    # Q's output where K or its output lies, and the reverse: 4 tokens, 28 heads and 4 heads of 256 bytes
    far = FAKE + (1 << 20)
    assert rot(k=far, ko=FAKE) == 2 and rot(k=far, ko=FAKE + 4 * 28 * 256 - 16) == 2
    assert rot(k=far, ko=far, qo=far + 4 * 4 * 256 - 16) == 2 and rot(k=far, ko=far, qo=far - 4 * 28 * 256 + 16) == 2
    assert make(theta=5e-324) == 2                                   # rates beyond what fp64 holds
    broken = binding._CRotaryPlan.from_buffer_copy(plan)
    broken.sections[1] = 23
    assert rot(plan=broken) == 2
    broken.sections[1], broken.pairing = 24, 5
    assert rot(plan=broken) == 2
    with pytest.raises(vs.VSError):
        vs.RotaryPlan(128, (16, 24, 23))


def test_rotary_refuses_outputs_over_the_positions():
    """A turned row over positions that other tokens still read.  4 tokens: 28 and 4 heads of 256 bytes, positions of 48."""
    L, s, plan = vs.lib(), _shape(), vs.RotaryPlan(128, (16, 24, 24)).c
    q, k, far = FAKE, FAKE + (1 << 20), FAKE + (2 << 20)
    nq, nk = 4 * 28 * 256, 4 * 4 * 256

    def rot(pos, qo, ko):
        return L.vs_rotary(ctypes.byref(s), ctypes.byref(plan), pos, 4, q if qo else None, k if ko else None, 0, qo, ko, None)

    for pos in (far, far + nq - 4, far - 44):
        assert rot(pos, far, k) == 2 and rot(pos, far, None) == 2
    for pos in (far, far + nk - 4, far - 44):
        assert rot(pos, q, far) == 2 and rot(pos, None, far) == 2
    assert rot(q + 64, q, k) == 2 and rot(k + 64, q, k) == 2              # rows turned in place


def test_cache8_sizes():
    s = _shape()
    assert vs.cache8_bytes(s, 1) == vs.cache8_bytes(s, 32) == 4 * 8320 and vs.cache8_bytes(s, 33) == 8 * 8320
    assert vs.cache8_bytes(s, 0) == 0 and vs.cache8_bytes(s, -5) == 0
    assert vs.cache8_bytes(_shape(4, 1, 64, vs.VS_F32), 32) == 0 and vs.cache8_bytes(_shape(4, 1, 128, vs.VS_F32), 32) == 0
    assert vs.cache8_bytes(_shape(d=64), 32) == 0 and vs.cache8_bytes(_shape(hq=5), 32) == 0
    assert vs.cache8_bytes(_shape(1, 1), 2 ** 31 - 1) == (2 ** 31 // 32) * 8320
    assert vs.cache8_bytes(_shape(4096, 4096), 2 ** 31 - 1) == 0       # beyond any memory
    need = [vs.cache8_workspace_bytes(s, t, 5000, 0) for t in (1, 16, 170, 171, 1000, 4096)]
    assert need[0] > 256
    for t, n in zip((1, 16, 170, 171, 1000), need):       # what serves a longer run serves a shorter one
        assert all(vs.cache8_workspace_bytes(s, m, 5000, 0) >= n for m in (t, t + 1, 170 + t, 4096))
        assert vs.cache8_workspace_bytes(s, t, 50, 0) <= n
    assert vs.cache8_workspace_bytes(s, 170, 5000, 16) >= vs.cache8_workspace_bytes(s, 170, 5000, 0)
    assert vs.cache8_workspace_bytes(s, 0, 0, 0) >= 256
    for bad in ((-1, 0, 0), (4097, 0, 0), (1, -1, 0), (1, 0, -1), (1, 0, 1025)):
        assert vs.cache8_workspace_bytes(s, *bad) == 0
    assert vs.cache8_workspace_bytes(_shape(4, 1, 64, vs.VS_F32), 4, 4, 1) == 0


@pytest.mark.parametrize("hq,hkv", [(28, 4), (24, 24), (8, 8), (8, 1), (5, 5)])
def test_a_workspace_serves_any_run_over_fewer_rows(hq, hkv):
    """The size is what the neediest run within the limits takes: it never falls as the limits go up."""
    s = _shape(hq, hkv)
    for tokens in (1, 9, 64, 107, 128, 300):
        sizes = [vs.cache8_workspace_bytes(s, tokens, 32 * b, 0) for b in range(80)]
        assert sizes == sorted(sizes), tokens
    for rows in (0, 300, 1000, 3000):
        sizes = [vs.cache8_workspace_bytes(s, t, rows, 0) for t in range(1, 400, 7)]
        assert sizes == sorted(sizes), rows


@pytest.mark.parametrize("hq,hkv", [(28, 4), (8, 8), (8, 1)])
def test_a_workspace_for_any_number_of_rows(hq, hkv):
    """Up to the largest number of rows that can be asked for."""
    s = _shape(hq, hkv)
    for tokens in (1, 37, 170, 4096):
        rows = [1000, 100_000, 2 ** 20, 2 ** 30, 2 ** 31 - 33, 2 ** 31 - 32, 2 ** 31 - 31, 2 ** 31 - 1]
        sizes = [vs.cache8_workspace_bytes(s, tokens, r, 0) for r in rows]
        assert sizes == sorted(sizes), (tokens, sizes)


def test_cache8_append_and_read_argument_errors():
    L, s = vs.lib(), _shape()

    def app(n=2, slab=FAKE, cap=64, lens=(5, 60), k=FAKE, v=FAKE, t=4, first=0, shape=s):
        arr = (ctypes.c_int32 * len(lens))(*lens)
        rc = L.vs_cache8_append(ctypes.byref(shape), n, slab, cap, arr, k, v, t, first, None)
        assert list(arr) == list(lens), "lengths changed by a refused call"
        return rc

    assert L.vs_cache8_append(ctypes.byref(s), 1, FAKE, 64, None, FAKE, FAKE, 4, 0, None) == 1
    assert app(slab=None) == 1 and app(k=None) == 1 and app(v=None) == 1
    assert app(n=0) == 2 and app(n=2 ** 20 + 1) == 2 and app(cap=0) == 2 and app(t=0) == 2
    assert app(first=-1) == 2 and app(first=4) == 2 and app(lens=(5, -1)) == 2
    assert app(lens=(5, 61)) == 4 and app(lens=(5, 64), first=3) == 4 and app(t=2 ** 31 - 1) == 4
    assert app(slab=ODD) == 6 and app(k=ODD) == 6 and app(v=ODD) == 6
    assert app(shape=_shape(4, 1, 64, vs.VS_F32)) == 3 and app(shape=_shape(hq=36)) == 3 and app(shape=_shape(hq=27)) == 2

    def read(n=2, slab=FAKE, cap=64, lens=(5, 60), firsts=(1, 3), rows=4, k=FAKE, v=FAKE, shape=s):
        return L.vs_cache8_read(ctypes.byref(shape), n, slab, cap, (ctypes.c_int32 * 2)(*lens),
                                None if firsts is None else (ctypes.c_int32 * 2)(*firsts), rows, k, v, None)

    assert read(slab=None) == 1 and read(k=None) == 1 and read(v=None) == 1
    assert read(n=0) == 2 and read(cap=0) == 2 and read(rows=0) == 2 and read(firsts=(-1, 0)) == 2 and read(lens=(-1, 4)) == 2
    assert read(firsts=(2, 3)) == 2 and read(firsts=(2 ** 31 - 1, 0)) == 2     # rows that are not there
    assert read(firsts=None, rows=6) == 2
    assert read(lens=(5, 65)) == 4
    assert read(slab=ODD) == 6 and read(k=ODD) == 6
    assert read(shape=_shape(4, 1, 64, vs.VS_F32)) == 3


def test_cache8_decode_argument_errors():
    L, s = vs.lib(), _shape()
    need = vs.cache8_workspace_bytes(s, 0, 0, 2)

    def dec(n=2, slab=FAKE, cap=8, lens=(5, 7), q=FAKE, kn=FAKE, vn=FAKE, out=FAKE, ws=FAKE, wsb=1 << 30, shape=s):
        arr = (ctypes.c_int32 * 2)(*lens)
        rc = L.vs_cache8_decode_attn(ctypes.byref(shape), n, slab, cap, arr, q, kn, vn, out, ws, wsb, None)
        assert list(arr) == list(lens)
        return rc

    assert dec(slab=None) == 1 and dec(q=None) == 1 and dec(out=None) == 1 and dec(kn=None) == 1 and dec(vn=None) == 1
    assert dec(n=0) == 2 and dec(n=1025) == 2 and dec(cap=0) == 2 and dec(lens=(-1, 5)) == 2
    assert dec(lens=(5, 8)) == 4 and dec(lens=(9, 8), kn=None, vn=None) == 4
    assert dec(lens=(0, 3), kn=None, vn=None) == 2                     # a stream with nothing to attend to
    assert dec(slab=ODD) == 6 and dec(q=ODD) == 6 and dec(out=ODD) == 6 and dec(vn=ODD) == 6 and dec(ws=ODD) == 6
    assert dec(ws=None) == 5 and dec(wsb=need - 512) == 5
    assert dec(shape=_shape(4, 1, 64, vs.VS_F32)) == 3


def test_cache8_prefill_argument_errors():
    L, s = vs.lib(), _shape()
    need = vs.cache8_workspace_bytes(s, 4, 5, 0)

    def pre(data=FAKE, cap=8, ln=5, q=FAKE, k=FAKE, v=FAKE, n=4, first=3, out=FAKE, ws=FAKE, wsb=1 << 30, shape=s):
        c = binding._CCache8(data, cap, ln)
        rc = L.vs_cache8_prefill_attn(ctypes.byref(shape), ctypes.byref(c), q, k, v, n, first, out, ws, wsb, None)
        assert c.len == ln
        return rc

    assert L.vs_cache8_prefill_attn(ctypes.byref(s), None, FAKE, FAKE, FAKE, 4, 3, FAKE, FAKE, 1 << 30, None) == 1
    assert pre(data=None) == 1 and pre(q=None) == 1 and pre(k=None) == 1 and pre(v=None) == 1 and pre(out=None) == 1
    assert pre(n=0, first=0) == 2 and pre(n=4097) == 2 and pre(first=-1) == 2 and pre(first=5) == 2 and pre(ln=-1) == 2 and pre(cap=-1) == 2
    assert pre(first=0) == 4 and pre(ln=8) == 4 and pre(ln=9, first=4) == 4
    assert pre(data=ODD) == 6 and pre(k=ODD) == 6 and pre(out=ODD) == 6 and pre(ws=ODD) == 6
    assert pre(ws=None) == 5 and pre(wsb=64) == 5 and need > 64
    assert pre(shape=_shape(4, 1, 64, vs.VS_F32)) == 3


# ---------------------------------------------------------------------------- what the binding refuses
def _refused(call, *args, **kwargs):
    with pytest.raises(vs.VSError) as err:
        call(*args, stream=0, **kwargs)
    assert err.value.code == 2


def test_binding_refuses_tensors_that_are_not_what_the_call_covers():
    """Memory that is smaller than the capacity says, fewer lengths than caches, tensors of other sizes, types and strides than the others': found
    before the library is called."""
    torch = pytest.importorskip("torch")
    s, n, cap, T = _shape(8, 2), 3, 40, 6
    lens = (ctypes.c_int32 * n)(4, 4, 4)

    def bf(*dims):
        return torch.zeros(dims, dtype=torch.bfloat16)

    slab, k, ws = torch.zeros((n, vs.cache8_bytes(s, cap)), dtype=torch.uint8), bf(n, T, 2, 128), torch.zeros(1 << 20, dtype=torch.uint8)
    few, wide = (ctypes.c_int32 * 2)(4, 4), bf(n, T, 2, 256)[..., :128]
    for bad in ((slab[:2], cap, lens, k, k), (slab, cap + 32, lens, k, k), (slab, cap, few, k, k), (slab, cap, lens, k, k[:, :5].contiguous()), (slab, cap, lens, k[..., :64].contiguous(), k),
                (slab, cap, lens, k.float(), k.float()), (slab, cap, lens, k, wide), (slab[:, ::2], cap, lens, k, k), (slab, cap, lens, k[:1].expand(n, T, 2, 128), k)):
        _refused(vs.cache8_append, s, *bad)
    for bad in ((slab[:2], cap, lens, None, k, k), (slab, cap, few, None, k, k), (slab, cap, lens, few, k, k), (slab, cap, lens, None, k, k[:2].contiguous()), (slab, cap, lens, None, wide, k)):
        _refused(vs.cache8_read, s, *bad)
    q, kn = bf(n, 8, 128), bf(n, 2, 128)
    for bad in ((slab[:2], cap, lens, q, kn, kn, q), (slab, 100, lens, q, kn, kn, q), (slab, cap, few, q, kn, kn, q), (slab, cap, lens, q, kn[:2], kn, q), (slab, cap, lens, q, kn, kn, q[:, :4].contiguous()),
                (slab, cap, lens, q, None, None, q.float()), (slab, cap, lens, bf(n, 2, 128), kn, kn, q)):
        _refused(vs.cache8_decode_attn, s, *bad, ws)
    cache, small, q, k = vs.Cache8(slab[0], cap, 4), vs.Cache8(slab[0], cap + 25, 4), bf(T, 8, 128), bf(T, 2, 128)
    for bad in ((small, q, k, k, q), (cache, q, k[:5], k, q), (cache, q, k, k.float(), q), (cache, q, k, k, q[:5]), (cache, q, bf(T, 2, 256)[..., :128], k, q)):
        _refused(vs.cache8_prefill_attn, s, *bad, ws)
    plan, pos = vs.RotaryPlan(128, (16, 24, 24)), torch.zeros((3, T), dtype=torch.int32)
    for bad in ((pos, q[:5], k, q, k), (pos, q, k, q, bf(T, 2, 64)), (pos[:, :5], q, k, q, k), (pos[:2], q, k, q, k), (pos, q, k.float(), q, k), (pos, q, None, bf(T, 8, 256)[..., :128], None),
                (torch.zeros((3, T + 1), dtype=torch.int32), q, k, q, k)):
        _refused(vs.rotary, s, plan, *bad)
    _refused(vs.cache8_append, s, slab, cap, lens, bf(n, T, 2, 128), bf(n, T + 1, 2, 128))       # caches that begin elsewhere in one of the two
    for bad in (pos.float(), pos.long()):
        with pytest.raises(AssertionError):
            vs.rotary(s, plan, bad, q, k, q, k, stream=0)
    # and what the library itself refuses still comes from there
    f32 = _shape(4, 1, 64, vs.VS_F32)
    with pytest.raises(vs.VSError) as err:
        vs.cache8_decode_attn(f32, slab, cap, lens, torch.zeros((n, 4, 64)), None, None, torch.zeros((n, 4, 64)), ws, stream=0)
    assert err.value.code == 3
    with pytest.raises(vs.VSError) as err:
        vs.cache8_append(s, slab, cap, lens, bf(n, 41, 2, 128), bf(n, 41, 2, 128), stream=0)
    assert err.value.code == 4 and list(lens) == [4] * n
