"""Linear attention with a fixed decay for each head, rotary positions and group norm, without a GPU: the oracle against
differences and identities, the frequencies' table against exact arithmetic, and every refusal of the entry points."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2607_11897_b200 as sfda
from oracle import operators as op
from paper_2607_11897_b200 import build as cuda_build


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return sfda.load()


def _difference(f, x, at, h=1e-6):
    y = np.array(x)
    y[at] += h
    up = f(y)
    y[at] -= 2 * h
    return (up - f(y)) / (2 * h)


def test_oracle_gradients_of_linear_attention_against_differences():
    rng = np.random.default_rng(0)
    B, T, H, Hk, dk, dv = 2, 5, 4, 2, 3, 2
    q, k, v = rng.normal(size=(B, T, H, dk)), rng.normal(size=(B, T, Hk, dk)), rng.normal(size=(B, T, Hk, dv))
    ld, lens, S0 = -rng.uniform(0, 1, H), [5, 3], rng.normal(size=(B, H, dk, dv))
    d_o, dS = rng.normal(size=(B, T, H, dv)), rng.normal(size=(B, H, dk, dv))

    def loss(**new):
        x = dict(q=q, k=k, v=v, S0=S0, **{}) | new
        o, S = op.linear_forward(x["q"], x["k"], x["v"], ld, lens, x["S0"], 0.7)
        return (o * d_o).sum() + (S * dS).sum()
    got = dict(zip(("q", "k", "v", "S0"), op.linear_backward(q, k, v, ld, d_o, dS, lens, S0, 0.7)))
    for name, x in (("q", q), ("k", k), ("v", v), ("S0", S0)):
        for _ in range(12):
            at = tuple(rng.integers(0, n) for n in x.shape)
            assert abs(got[name][at] - _difference(lambda y: loss(**{name: y}), x, at)) < 1e-7, (name, at)
    assert not got["q"][1, 3:].any() and not got["k"][1, 3:].any()


def test_oracle_of_linear_attention_against_explicit_sums():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(1, 7, 1, 3)), rng.normal(size=(1, 7, 1, 3)), rng.normal(size=(1, 7, 1, 2))
    o, S = op.linear_forward(q, k, v, [-0.3])
    for t in range(7):
        want = sum(np.exp(-0.3 * (t - i)) * (q[0, t, 0] @ k[0, i, 0]) * v[0, i, 0] for i in range(t + 1))
        assert np.abs(o[0, t, 0] - want).max() < 1e-12
    alone, _ = op.linear_forward(q, k, v, [-np.inf])
    assert np.allclose(alone[0, :, 0], (q[0, :, 0] * k[0, :, 0]).sum(-1, keepdims=True) * v[0, :, 0])


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_oracle_gradients_of_group_norm_against_differences(silu, gated):
    rng = np.random.default_rng(2)
    x, w, b, dy = rng.normal(size=(3, 12)), rng.normal(size=12), rng.normal(size=12), rng.normal(size=(3, 12))
    gate = rng.normal(size=(3, 12)) if gated else None
    dx, dw, db, dgate = op.group_norm_backward(x, w, b, gate, dy, 3, 1e-2, silu)
    f = lambda **n: (op.group_norm(**(dict(x=x, weight=w, bias=b, gate=gate) | n), groups=3, eps=1e-2, silu=silu) * dy).sum()  # noqa: E731
    for name, value, got in (("x", x, dx), ("weight", w, dw), ("bias", b, db), ("gate", gate, dgate)):
        if value is None:
            continue
        for at in np.ndindex(value.shape):
            assert abs(got[at] - _difference(lambda y: f(**{name: y}), value, at)) < 1e-7, (name, at)


def test_oracle_rotations_keep_the_norm_and_depend_on_the_distance():
    rng = np.random.default_rng(3)
    x, y, f = rng.normal(size=(1, 1, 1, 8)), rng.normal(size=(1, 1, 1, 8)), op.rotary_frequencies(6)
    for halves in (False, True):
        a, b = op.rotary(x, [[11]], f, halves), op.rotary(y, [[4]], f, halves)
        assert abs((a * b).sum() - (op.rotary(x, [[107]], f, halves) * op.rotary(y, [[100]], f, halves)).sum()) < 1e-12
        assert np.allclose(op.rotary(a, [[11]], f, halves, inverse=True), x) and np.array_equal(a[..., 6:], x[..., 6:])


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "parts"])
@pytest.mark.parametrize("rot", [4, 62, 128])
def test_turns_are_the_frequencies_to_the_last_bits_of_a_double(lib, scaling, rot):
    code = dict(plain=sfda.SFDA_ROTARY_PLAIN, linear=sfda.SFDA_ROTARY_LINEAR, base=sfda.SFDA_ROTARY_BASE, parts=sfda.SFDA_ROTARY_PARTS)
    got = sfda.sfda_rotary_turns(rot, 10000.0, code[scaling], 8.0, 1.0, 4.0, 4096.0).numpy().view(np.uint64)
    want = op.rotary_frequencies(rot, 10000.0, scaling, 8.0, 1.0, 4.0, 4096.0) / (2 * np.pi) * 2.0 ** 64
    assert got.shape == (rot // 2,)
    # the oracle's doubles carry a few roundings of 2^-53 (the power's exponent times ln base, up to 9.2, among them), and a
    # count is a whole number: half a count of rounding, which is 2^-46 of the slowest pair's 3.7e13 counts here
    for g, w in zip(got, want):
        assert abs(Fraction(int(g)) - Fraction(w)) <= Fraction(1, 2) + Fraction(w) * 32 / 2 ** 53


def test_turns_refuse_what_has_no_frequencies(lib):
    for bad, status in ((dict(rot=3), -2), (dict(rot=0), -2), (dict(rot=8, base=1.0), -8), (dict(rot=8, base=float("nan")), -8),
                        (dict(rot=8, scaling=9), -8), (dict(rot=8, scaling=1, factor=0.5), -8),
                        (dict(rot=2, scaling=2, factor=2.0), -2), (dict(rot=8, scaling=3, factor=2.0, low=4.0, high=4.0), -8),
                        (dict(rot=8, scaling=3, factor=2.0, trained=0.0), -8)):
        with pytest.raises(sfda.SfdaError) as e:
            sfda.sfda_rotary_turns(**bad)
        assert e.value.status == status, bad
    assert lib.sfda_rotary_turns(None, 8, 1e4, 0, 1.0, 1.0, 4.0, 1.0) == -1


vp = ctypes.c_void_p
OK = vp(0x1000)                       # never dereferenced: validation fails first
OFF = vp(0x1004)
WS = vp(0x2000)


def test_linear_entry_points_validate_on_the_host(lib):
    f = lambda p, d, scale=1.0, ws=WS, n=1 << 40: lib.sfda_linear_forward(*p, *d, scale, ws, n, None)  # noqa: E731
    p, d = [OK] * 4 + [None, None, OK, None], [1, 64, 4, 2, 128, 128, 1]
    for i in (0, 1, 2, 3, 6):
        assert f(p[:i] + [None] + p[i + 1:], d) == -1
    for i, bad in ((0, 0), (1, 0), (2, 0), (3, 0), (3, 3), (3, 8), (4, 127)):
        assert f(p, d[:i] + [bad] + d[i + 1:]) == -2, (i, bad)
    for i, bad in ((4, 96), (5, 32), (6, 2)):
        assert f(p, d[:i] + [bad] + d[i + 1:]) == -3, (i, bad)
    for i in range(8):
        assert f(p[:i] + [OFF] + p[i + 1:], d) == -4
    assert f(p, d, ws=OFF) == -4
    assert f(p, d, float("nan")) == -8 and f(p, d, float("inf")) == -8
    need = lib.sfda_linear_workspace_bytes(*d)
    if need:
        assert f(p, d, ws=None, n=0) == -5 and f(p, d, n=need - 1) == -5
    assert lib.sfda_linear_workspace_bytes(1, 64, 4, 3, 128, 128, 1) == 0

    g = lambda p, d, scale=1.0, ws=WS, n=1 << 40: lib.sfda_linear_backward(*p, *d, scale, ws, n, None)  # noqa: E731
    p = [OK] * 4 + [None, None, OK, None] + [vp(0x3000)] * 4
    for i in (0, 1, 2, 3, 6, 8, 9, 10, 11):
        assert g(p[:i] + [None] + p[i + 1:], d) == -1
    assert g(p, d[:3] + [3] + d[4:]) == -2 and g(p, d[:4] + [32] + d[5:]) == -3
    for i in range(12):
        assert g(p[:i] + [OFF] + p[i + 1:], d) == -4
    assert g(p[:7] + [p[11]] + p[8:], d) == -8                            # dS_T is what dS0 would overwrite
    assert g(p, d, float("-inf")) == -8
    need = lib.sfda_linear_backward_workspace_bytes(*d)
    assert need >= 64 * 4 * 256 * 4                                       # shared heads: every query head's gradients
    assert g(p, d, ws=None, n=0) == -5 and g(p, d, n=need - 1) == -5

    h = lambda p, d, scale=1.0: lib.sfda_linear_step(*p, *d, scale, None)  # noqa: E731
    p, d = [OK] * 6, [1, 4, 2, 128, 128, 1]
    for i in range(6):
        assert h(p[:i] + [None] + p[i + 1:], d) == -1 and h(p[:i] + [OFF] + p[i + 1:], d) == -4
    assert h(p, [0] + d[1:]) == -2 and h(p, d[:2] + [3] + d[3:]) == -2 and h(p, d[:3] + [96, 128, 1]) == -3
    assert h(p, d, float("nan")) == -8


def test_rotary_validates_on_the_host(lib):
    def f(p=(OK,) * 6, B=1, T=1, H=2, H_kv=2, d=64, rot=64, s=(128, 128, 128, 128), layout=0, amp=1.0, dtype=1):
        return lib.sfda_rotary(*p, B, T, H, H_kv, d, rot, *s, layout, amp, 0, dtype, None)
    p = [OK] * 6
    for i in range(6):                                                    # of q, k, positions, turns, q_out, k_out
        assert f(p[:i] + [None] + p[i + 1:]) == -1 and f(p[:i] + [OFF] + p[i + 1:]) == -4
    for bad in (dict(B=0), dict(T=0), dict(H=0), dict(H_kv=0), dict(d=63, rot=2), dict(d=1026, rot=2), dict(rot=65), dict(rot=66),
                dict(rot=-2), dict(s=(126, 128, 128, 128)), dict(s=(128, 64, 128, 128)), dict(s=(128, 128, 128, 129)),
                dict(s=(-128, 128, 128, 128))):
        assert f(**bad) == -2, bad
    assert f(dtype=2) == -3 and f(layout=2) == -8 and f(amp=float("nan")) == -8


def test_group_norm_validates_on_the_host(lib):
    f = lambda p, rows=4, C=64, G=2, eps=1e-5, act=1, dt=1: lib.sfda_group_norm(*p, rows, C, G, eps, act, dt, None)  # noqa: E731
    p = [OK, None, None, None, OK]
    assert f([None] + p[1:]) == -1 and f(p[:4] + [None]) == -1
    assert f(p, rows=0) == -2 and f(p, C=0) == -2 and f(p, G=0) == -2 and f(p, G=3) == -2
    assert f(p, dt=3) == -3 and f(p, act=2) == -8
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert f(p, eps=eps) == -8
    for i in range(5):
        assert f(p[:i] + [OFF] + p[i + 1:]) == -4
    assert f(p, C=70000 * 5000, G=70000) == -3                            # more groups wider than a warp than a grid has rows
    g = lambda p, ws=WS, n=1 << 40, rows=4, C=64: lib.sfda_group_norm_backward(*p, rows, C, 2, 1e-5, 1, 1, ws, n, None)  # noqa: E731
    p = [OK, OK, OK, OK, OK, OK, OK, OK, OK]
    for i in (0, 4, 5, 8):
        assert g(p[:i] + [None] + p[i + 1:]) == -1
    for i in range(9):
        assert g(p[:i] + [OFF] + p[i + 1:]) == -4
    need = lib.sfda_group_norm_backward_workspace_bytes(4, 64)
    assert need >= 2 * 4 * 64 and g(p, None, 0) == -5 and g(p, n=need - 1) == -5
    assert lib.sfda_group_norm_backward_workspace_bytes(0, 64) == 0


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    x = torch.zeros(1, 1, 2, 64)
    with pytest.raises(ValueError):
        sfda.sfda_linear_forward(x, x, x, torch.zeros(2), None, None, x, None)
    with pytest.raises(ValueError):
        sfda.sfda_linear_step(x[0], x[0], x[0], torch.zeros(2), torch.zeros(1, 2, 64, 64), x[0])
    with pytest.raises(ValueError):
        sfda.sfda_rotary(x, None, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(32, dtype=torch.int64), x, None)
    with pytest.raises(ValueError):
        sfda.sfda_group_norm(x, None, None, None, x, 1)
