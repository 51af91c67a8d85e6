"""Calls of the operators beside the recurrence that their documentation allows and that are easy to get wrong: inputs that share an
address, values and parameters that are extreme or not finite, groups of one value, named streams, waits that run out."""
import numpy as np
import pytest
import torch

import paper_2607_11897_b200 as sfda
from oracle import operators as op

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def scratch(n):
    return torch.empty(n, device="cuda", dtype=torch.uint8) if n else None


# ---- linear attention: inputs that begin at the same address -------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_k,d_v", [(64, 128), (128, 64), (64, 64), (128, 128)])
@pytest.mark.parametrize("pair", ["kv", "qv", "qk", "qd"])
def test_linear_inputs_may_be_views_of_one_buffer(pair, d_k, d_v, dtype):
    """Only outputs may not overlap inputs.  Two inputs that begin at the same address, of the same number of heads and of equal or
    different widths, give the bits that they give as tensors of their own."""
    B, T, H, dt = 2, 200, 3, DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(1)
    width = dict(q=d_k, k=d_k, v=d_v, d=d_v)
    alone = {n: torch.randn(B, T, H, w, device="cuda", generator=g).to(dt) for n, w in width.items()}
    buffer = torch.randn(B * T * H * max(d_k, d_v), device="cuda", generator=g).to(dt)
    views = dict(alone)
    for n in pair:
        views[n] = buffer[:B * T * H * width[n]].view(B, T, H, width[n])
        alone[n] = views[n].clone()
    assert views[pair[0]].data_ptr() == views[pair[1]].data_ptr() and alone[pair[0]].data_ptr() != alone[pair[1]].data_ptr()
    ld, sizes = -torch.rand(H, device="cuda", generator=g), (B, T, H, H, d_k, d_v, int(dtype == "bf16"))

    def run(x):
        o, S = torch.empty(B, T, H, d_v, device="cuda", dtype=dt), torch.empty(B, H, d_k, d_v, device="cuda")
        sfda.sfda_linear_forward(x["q"], x["k"], x["v"], ld, None, None, o, S, 0.5, scratch(sfda.sfda_linear_workspace_bytes(*sizes)))
        grads = [torch.empty(B, T, H, w, device="cuda", dtype=dt) for w in (d_k, d_k, d_v)] + [torch.empty_like(S)]
        sfda.sfda_linear_backward(x["q"], x["k"], x["v"], ld, None, None, x["d"], None, *grads, 0.5,
                                  scratch(sfda.sfda_linear_backward_workspace_bytes(*sizes)))
        return [o, S] + grads

    for name, a, b in zip(("o", "S_T", "dq", "dk", "dv", "dS0"), run(views), run(alone)):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("d_k,d_v", [(64, 64), (128, 128)])
def test_linear_fp32_keeps_the_bits_of_its_operands(d_k, d_v):
    """Root mean squares, relative: an operand's low tf32 part (2^-11 of it at most, 2^-12.2 in the mean) is cut at 2^-10 of itself, so 1e-7 for
    each of two operands; a product of two low parts that is left out, 4e-8; sums in accumulators, cut off at each of up to 16 steps
    by half a unit on average, at most 16 x 2^-25 = 5e-7 where all steps are of full size, half of that on the way to it.  Two
    products in a row: under 6e-7, and 1e-6 with the fp32 additions and powers around them."""
    B, T, H = 1, 700, 4
    g = torch.Generator(device="cuda").manual_seed(9)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, d_o, S0, dS = r(B, T, H, d_k), r(B, T, H, d_k), r(B, T, H, d_v), r(B, T, H, d_v), r(B, H, d_k, d_v), r(B, H, d_k, d_v)
    ld = torch.tensor([-1.0, -0.05, -2.0 ** -8, -2.0 ** -12], device="cuda")
    o, S, grads = torch.empty_like(v), torch.empty_like(S0), [torch.empty_like(t) for t in (q, k, v, S0)]
    sfda.sfda_linear_forward(q, k, v, ld, None, S0, o, S, 0.5)
    sfda.sfda_linear_backward(q, k, v, ld, None, S0, d_o, dS, *grads, 0.5)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = (*op.linear_forward(f(q), f(k), f(v), f(ld), None, f(S0), 0.5), *op.linear_backward(f(q), f(k), f(v), f(ld), f(d_o), f(dS), None, f(S0), 0.5))
    for name, got, y in zip(("o", "S_T", "dq", "dk", "dv", "dS0"), [o, S] + grads, want):
        assert np.linalg.norm(f(got) - y) <= 1e-6 * np.linalg.norm(y), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_linear_largest_finite_values_do_not_reach_earlier_tokens(sign, dtype):
    """The type's largest and lowest value in v, q and d_o: masked scores are zeros of a dense product, and zero times it is zero.  What does
    not depend on the entry has the bits of the clean run."""
    T, t, c, dt = 300, 140, 17, DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(7)
    clean = {n: torch.randn(1, T, 2, 64, device="cuda", generator=g).to(dt) for n in "qkvd"}
    ld, sizes = torch.tensor([-0.01, -0.7], device="cuda"), (1, T, 2, 2, 64, 64, int(dtype == "bf16"))

    def run(x):
        o, S = torch.empty_like(x["v"]), torch.empty(1, 2, 64, 64, device="cuda")
        sfda.sfda_linear_forward(x["q"], x["k"], x["v"], ld, None, None, o, S, 0.5, scratch(sfda.sfda_linear_workspace_bytes(*sizes)))
        grads = [torch.empty_like(x["q"]) for _ in range(3)] + [torch.empty_like(S)]
        sfda.sfda_linear_backward(x["q"], x["k"], x["v"], ld, None, None, x["d"], None, *grads, 0.5,
                                  scratch(sfda.sfda_linear_backward_workspace_bytes(*sizes)))
        return [o, S] + grads

    want = run(clean)
    for h in (0, 1):
        for name in "vqd":
            x = dict(clean)
            x[name] = clean[name].clone()
            x[name][0, t, h, c] = sign * torch.finfo(dt).max
            reach = [torch.zeros_like(y, dtype=torch.bool) for y in want]
            o, S, dq, dk, dv, dS = reach
            if name == "v":
                o[0, t:, h, c] = S[0, h, :, c] = dq[0, t:, h] = dk[0, t, h] = True
            elif name == "q":
                o[0, t, h] = dk[0, :t + 1, h, c] = dv[0, :t + 1, h] = dS[0, h, c] = True
            else:
                dq[0, t, h] = dk[0, :t + 1, h] = dv[0, :t + 1, h, c] = dS[0, h, :, c] = True
            for n, (got, y, r) in enumerate(zip(run(x), want, reach)):
                assert torch.equal(got[~r], y[~r]), (name, h, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T,t", [(300, 140), (2500, 1500)])
def test_linear_values_that_are_not_finite_at_weak_decays_and_in_cut_sequences(T, t, value, dtype):
    """Heads that hardly forget, whose scores the bf16 kernel scales by the column, and sequences that it cuts into stretches."""
    c, dt = 17, DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(8)
    clean = {n: torch.randn(1, T, 2, 64, device="cuda", generator=g).to(dt) for n in "qkvd"}
    clean["k"] = (0.1 * clean["k"]).to(dt)
    ld, sizes = torch.tensor([-0.01, 0.0], device="cuda"), (1, T, 2, 2, 64, 64, int(dtype == "bf16"))
    S0 = torch.randn(1, 2, 64, 64, device="cuda", generator=g)

    def run(x):
        o, S = torch.empty_like(x["v"]), torch.empty_like(S0)
        sfda.sfda_linear_forward(x["q"], x["k"], x["v"], ld, None, S0, o, S, 0.5, scratch(sfda.sfda_linear_workspace_bytes(*sizes)))
        grads = [torch.empty_like(x["q"]) for _ in range(3)] + [torch.empty_like(S)]
        sfda.sfda_linear_backward(x["q"], x["k"], x["v"], ld, None, S0, x["d"], S0, *grads, 0.5,
                                  scratch(sfda.sfda_linear_backward_workspace_bytes(*sizes)))
        return [o, S] + grads

    want = run(clean)
    for h in (0, 1):
        for name in "qkvd":
            x = dict(clean)
            x[name] = clean[name].clone()
            x[name][0, t, h, c] = value
            reach = [torch.zeros_like(y, dtype=torch.bool) for y in want]
            o, S, dq, dk, dv, dS = reach
            if name == "q":
                o[0, t, h] = dk[0, :t + 1, h, c] = dv[0, :t + 1, h] = dS[0, h, c] = True
            elif name == "k":
                o[0, t:, h] = S[0, h, c] = dq[0, t:, h, c] = dv[0, t, h] = True
            elif name == "v":
                o[0, t:, h, c] = S[0, h, :, c] = dq[0, t:, h] = dk[0, t, h] = True
            else:
                dq[0, t, h] = dk[0, :t + 1, h] = dv[0, :t + 1, h, c] = dS[0, h, :, c] = True
            for n, (got, y, r) in enumerate(zip(run(x), want, reach)):
                assert torch.equal(got[~r], y[~r]), (name, h, n)
                assert not torch.isfinite(got[r]).any(), (name, h, n)


# ---- group norm ------------------------------------------------------------------------------------------------------
def norm_inputs(rows, C, dtype, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return (r(rows, C) + mean).to(DTYPES[dtype]), r(C), r(C), r(rows, C).to(DTYPES[dtype]), r(rows, C).to(DTYPES[dtype])


def norm(x, w, b, gate, dy, groups, eps, act):
    """(y, dx, dweight, dbias, dgate)"""
    e, C = torch.empty_like, x.shape[1]
    y, dx, dw, db, dg = e(x), e(x), e(w), e(w), None if gate is None else e(x)
    sfda.sfda_group_norm(x, w, b, gate, y, groups, eps, act)
    sfda.sfda_group_norm_backward(x, w, b, gate, dy, dx, dw, db, dg, groups, eps, act,
                                  scratch(sfda.sfda_group_norm_backward_workspace_bytes(x.shape[0], C)))
    return y, dx, dw, db, dg


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("C,groups", [(288, 3), (252, 7), (1500, 3), (2 * 1100, 2), (2 * 5003, 2), (256, 2)])
def test_group_norm_parameters_that_are_not_finite_stay_in_their_group(C, groups, gated, act, dtype):
    """The first channel's weight or bias is not finite: results of the other groups keep their bits, whether or not a group fills
    the lanes that work on it."""
    x, w, b, gate, dy = norm_inputs(5, C, dtype, 2)
    gate = gate if gated else None
    D, clean = C // groups, norm(x, w, b, gate, dy, groups, 1e-5, act)
    for value in (float("inf"), float("nan")):
        for which in (0, 1):
            params = [w.clone(), b.clone()]
            params[which][0] = value
            for name, got, want in zip(("y", "dx", "dweight", "dbias", "dgate"), norm(x, *params, gate, dy, groups, 1e-5, act), clean):
                if want is not None:
                    assert torch.equal(got[..., D:], want[..., D:]), (name, value, which)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("D", [36, 96, 100, 128, 129, 500, 5003])
def test_group_norm_of_constant_groups_is_the_bias_at_any_width(D, eps, dtype):
    """A group of one value has no deviation, however large the value and small eps.  bf16: a sum of D equal values is exact (8 + 13
    bits), and so is the mean.  fp32: the sum is off by its roundings, so that all differences are the same j units in the last place
    of the value, j < 100 (45 additions in a row at most, half a unit each, in a binade that may be half as wide); D j < 2^24, so
    their own mean is exact and what is left is zero."""
    g = torch.Generator(device="cuda").manual_seed(D)
    c = torch.exp(torch.rand(64, 2, 1, device="cuda", generator=g) * 23.0 - 11.5) * (torch.randint(0, 2, (64, 2, 1), device="cuda", generator=g) * 2 - 1)
    x = c.expand(64, 2, D).reshape(64, 2 * D).to(DTYPES[dtype])
    w, b = torch.randn(2 * D, device="cuda", generator=g), torch.randn(2 * D, device="cuda", generator=g)
    y = torch.empty_like(x)
    sfda.sfda_group_norm(x, w, b, None, y, 2, eps)
    assert torch.equal(y, b.to(x.dtype).expand(64, 2 * D))
    # n = 0: dweight vanishes, dx = (dn - mean of dn) / sqrt(eps)
    dy = torch.randn(64, 2 * D, device="cuda", generator=g).to(x.dtype)
    _, dx, dw, db, _ = norm(x, w, b, None, dy, 2, eps, 0)
    assert not dw.any()
    dn = (dy.double() * w.double()).view(64, 2, D)
    want = ((dn - dn.mean(-1, keepdim=True)) / eps ** 0.5).view(64, 2 * D)
    # a mean and three operations in fp32: 2e-6, as for all shapes; one rounding of half a step for bf16
    assert (dx.double() - want).norm() / want.norm() <= (2e-6 if dtype == "f32" else torch.finfo(torch.bfloat16).eps / 2)


def test_group_norm_of_a_variance_below_its_rounding_is_finite():
    """The variance about the first mean is less than that about the true one by the square of the means' distance.  Where nearly all
    of it is that distance (groups of one value, or of one value but for one unit in the last place), rounding may leave less than
    nothing, and an eps of 1e-12 does not lift it above zero."""
    g = torch.Generator(device="cuda").manual_seed(6)
    for rows, D in ((4096, 500), (4096, 1000), (64, 1 << 18)):
        c = torch.exp(torch.rand(rows, 1, device="cuda", generator=g) * 6.9 + 6.9).expand(rows, D).contiguous()
        one = c.clone()
        one[:, D // 3] = torch.nextafter(one[:, D // 3], torch.full((), float("inf"), device="cuda"))
        for x in (c, one):
            y = torch.empty_like(x)
            sfda.sfda_group_norm(x, None, None, None, y, 1, 1e-12)
            assert torch.isfinite(y).all(), (rows, D)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("D", [36, 100, 128, 500, 2048, 5003])
def test_group_norm_of_unit_deviations_about_a_large_mean(D, gated):
    """Deviations of 1 about 4096 in fp32, the forward and the gradients.  Differences from the first mean are exact (multiples of 2^-12
    below 2^3), and their own mean takes off what that one's rounding (up to some 2^-12) left: so what holds for a mean of 0
    holds here, a sum and a dozen operations in fp32, 2e-6.  Without the second mean n is off by about 1e-4."""
    x, w, b, gate, dy = norm_inputs(20, 2 * D, "f32", 3, mean=4096.0)
    gate = gate if gated else None
    f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    want = (op.group_norm(f(x), f(w), f(b), f(gate), 2, 1e-5, True), *op.group_norm_backward(f(x), f(w), f(b), f(gate), f(dy), 2, 1e-5, True))
    # (sums over rows partly cancel: four times as much, as for all shapes)
    for name, got, y, t in zip(("y", "dx", "dweight", "dbias", "dgate"), norm(x, w, b, gate, dy, 2, 1e-5, 1), want, (2e-6, 2e-6, 8e-6, 8e-6, 2e-6)):
        if y is not None:
            assert np.linalg.norm(f(got) - y) <= t * np.linalg.norm(y), name


# ---- named streams -----------------------------------------------------------------------------------------------------
B, T, H, D = 2, 150, 4, 64


def stream_calls():
    """name: (inputs, outputs, call): every entry point that enqueues work, on given inputs and outputs and a stream."""
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    q, k, v, d_o = (r(B, T, H, D) for _ in range(4))
    ld, w, b = -torch.rand(H, device="cuda", generator=g), torch.randn(H * D, device="cuda", generator=g), torch.randn(H * D, device="cuda", generator=g)
    state = torch.randn(B, H, D, D, device="cuda", generator=g)
    pos, turns = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1), sfda.sfda_rotary_turns(D).cuda()
    e, sizes = torch.empty_like, (B, T, H, H, D, D, sfda.SFDA_BF16)
    fws, bws = scratch(sfda.sfda_linear_workspace_bytes(*sizes)), scratch(sfda.sfda_linear_backward_workspace_bytes(*sizes))
    x, gate, dy = (t.view(B * T, H * D) for t in (q, k, v))
    nws = scratch(sfda.sfda_group_norm_backward_workspace_bytes(B * T, H * D))
    one = [t[:, 0].contiguous() for t in (q, k, v)]
    return {
        "linear_forward": ([q, k, v, state], [e(q), e(state)],
                           lambda i, o, s: sfda.sfda_linear_forward(*i[:3], ld, None, i[3], *o, 0.5, fws, s)),
        "linear_backward": ([q, k, v, state, d_o], [e(q), e(k), e(v), e(state)],
                            lambda i, o, s: sfda.sfda_linear_backward(*i[:3], ld, None, i[3], i[4], None, *o, 0.5, bws, s)),
        "linear_step": (one + [state], [e(one[0])], lambda i, o, s: sfda.sfda_linear_step(*i[:3], ld, i[3], o[0], 0.5, s)),
        "rotary": ([q, k], [e(q), e(k)], lambda i, o, s: sfda.sfda_rotary(*i, pos, turns, *o, 0, 1.0, False, s)),
        "group_norm": ([x, gate], [e(x)], lambda i, o, s: sfda.sfda_group_norm(i[0], w, b, i[1], o[0], H, 1e-5, 1, s)),
        "group_norm_backward": ([x, gate, dy], [e(x), e(w), e(w), e(x)],
                                lambda i, o, s: sfda.sfda_group_norm_backward(i[0], w, b, i[1], i[2], *o, H, 1e-5, 1, nws, s)),
    }


@pytest.mark.parametrize("name", ["linear_forward", "linear_backward", "linear_step", "rotary", "group_norm", "group_norm_backward"])
def test_calls_wait_for_the_stream_that_is_named(name):
    """The stream is held up before it writes the inputs; a call on it sees them, one that went to the current stream would read what
    lay there before.  Outputs, inputs and scratch are made, and the device is idle, before the stream is held up, and all stay alive
    until it is done."""
    values, out, call = stream_calls()[name]
    inputs = [t.clone() for t in values]
    call(inputs, out, None)
    want = [t.clone() for t in inputs + out]
    for t in inputs:
        t.fill_(7.0)
    for t in out:
        t.fill_(-3.0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(40_000_000)                            # 20 ms or more
        for t, y in zip(inputs, values):
            t.copy_(y)
    assert torch.cuda.current_stream() != s and not s.query()
    call(inputs, out, s)
    assert not s.query()
    s.synchronize()
    for a, b in zip(inputs + out, want):
        assert torch.equal(a, b)


# ---- waits that run out ------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def development():
    from paper_2607_11897_b200 import binding
    from paper_2607_11897_b200 import build as cuda_build
    return binding.load_library(cuda_build.build_variant("chaos", ["-DSFDA_WS_CHAOS"]))


# barriers that warps arrive at (their places in sfda_linear_tc.cu): the output's place, the keys, P, the output in tensor memory and in
# shared memory, the state, and e of heads that forget fast
@pytest.mark.parametrize("barrier", [6, 9, 11, 13, 14, 15, 16])
@pytest.mark.parametrize("sizes", [(3, 300, 6, 6, 128, 128), (1, 4000, 2, 1, 128, 128), (2, 400, 4, 2, 64, 128)])
def test_linear_waits_that_run_out_are_reported_and_leave_the_context_usable(development, monkeypatch, sizes, barrier):
    """The bf16 kernel of a development build with one of its roles' arrivals withheld and a limit of milliseconds: all roles leave, the
    kernel ends, the status says so, of whole and of cut sequences (two launches) and of gradients.  The same call with the
    plain build and the same workspace gives its bits again and clears the status."""
    from paper_2607_11897_b200 import binding
    B, T, H, H_kv, d_k, d_v = sizes
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, d_o = r(B, T, H, d_k).bfloat16(), (0.1 * r(B, T, H_kv, d_k)).bfloat16(), r(B, T, H_kv, d_v).bfloat16(), r(B, T, H, d_v).bfloat16()
    ld, S0 = torch.tensor([-0.001, -0.9, -0.1, -30.0, 0.0, -0.3][:H], device="cuda"), r(B, H, d_k, d_v)
    size = sizes + (sfda.SFDA_BF16,)
    fws, bws = scratch(sfda.sfda_linear_workspace_bytes(*size)), scratch(sfda.sfda_linear_backward_workspace_bytes(*size))

    def run():
        o, S, grads = torch.zeros_like(d_o), torch.zeros_like(S0), [torch.zeros_like(t) for t in (q, k, v, S0)]
        sfda.sfda_linear_forward(q, k, v, ld, None, S0, o, S, 0.5, fws)
        sfda.sfda_linear_backward(q, k, v, ld, None, S0, d_o, None, *grads, 0.5, bws)
        torch.cuda.synchronize()
        return [o, S] + grads

    want = run()
    with monkeypatch.context() as m:
        m.setattr(binding, "_LIB", development)
        m.setenv("SFDA_WITHHOLD_LINEAR", str(barrier))
        run()
        for ws in (fws, bws):
            with pytest.raises(sfda.SfdaError) as e:
                sfda.sfda_workspace_status(ws)
            assert e.value.status == -7
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
        assert sfda.sfda_workspace_status(fws) == 0 and sfda.sfda_workspace_status(bws) == 0
