"""Linear attention with a fixed decay for each head, rotary positions and group norm on the GPU, through the binding, against
the oracle in 64 bits.

Tolerances are relative 2-norms.  fp32 outputs: operands in two tf32 parts lose at most 2^-22 each (twice per product, two
products in a row), sums of a few hundred terms in fp32 as much again: 4e-6.  bf16 outputs are rounded once, and on the way the
bf16 kernels round the masked scores and the state's copy for the products once each: three roundings of at most half a step
(eps / 2), each of root mean square (eps / 2) / sqrt(3), added without taking them for independent.  States of bf16 calls hold
products whose one factor is in two bf16 parts (2^-17), summed in fp32: 1e-5."""
import numpy as np
import pytest
import torch

import paper_2607_11897_b200 as sfda
from oracle import operators as op

pytestmark = pytest.mark.gpu
BF16 = 3 * (torch.finfo(torch.bfloat16).eps / 2) / 3 ** 0.5
F32, STATE = 4e-6, 1e-5
ROUND = torch.finfo(torch.bfloat16).eps / 2
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def off(x, y):
    x, y = x.detach().double().cpu().numpy() if torch.is_tensor(x) else x, np.asarray(y, np.float64)
    n = np.linalg.norm(y)
    return np.linalg.norm(x - y) / n if n else np.linalg.norm(x)


def tol(dtype, state=False):
    return F32 if dtype == torch.float32 else STATE if state else BF16


class Linear:
    """One set of inputs, the calls on it and the oracle's answers."""

    def __init__(self, B, T, H, H_kv=None, dk=128, dv=128, dtype="bf16", decay=None, lens=None, state=True, seed=0, scale=0.3):
        H_kv, dt = H_kv or H, DTYPES[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.sizes = (B, T, H, H_kv, dk, dv)
        self.q, self.v = r(B, T, H, dk).to(dt), r(B, T, H_kv, dv).to(dt)
        k = r(B, T, H_kv, dk)
        self.k = (k / k.norm(dim=-1, keepdim=True)).to(dt)
        if decay is None:
            decay = [-(2.0 ** -(i % 8)) for i in range(H)]
        self.log_decay = torch.tensor(decay, device="cuda", dtype=torch.float32)
        self.lens = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
        self.S0 = r(B, H, dk, dv) * 0.1 if state else None
        self.d_o, self.dS_T = r(B, T, H, dv).to(dt), r(B, H, dk, dv) if state else None
        self.scale, self.dt = scale, dt

    def code(self):
        return sfda.SFDA_BF16 if self.dt == torch.bfloat16 else sfda.SFDA_F32

    def workspace(self, backward=False):
        n = (sfda.sfda_linear_backward_workspace_bytes if backward else sfda.sfda_linear_workspace_bytes)(*self.sizes, self.code())
        return torch.empty(n, device="cuda", dtype=torch.uint8) if n else None

    def forward(self, ws="own", fill=0.0, stream=None):
        B, T, H, H_kv, dk, dv = self.sizes
        o = torch.full((B, T, H, dv), fill, device="cuda", dtype=self.dt)
        S_T = torch.full((B, H, dk, dv), float("nan"), device="cuda")
        sfda.sfda_linear_forward(self.q, self.k, self.v, self.log_decay, self.lens, self.S0, o, S_T, self.scale,
                                 self.workspace() if ws == "own" else ws, stream)
        return o, S_T

    def backward(self, ws="own", fill=0.0, stream=None):
        B, T, H, H_kv, dk, dv = self.sizes
        out = [torch.full_like(x, fill) for x in (self.q, self.k, self.v)] + [torch.full((B, H, dk, dv), float("nan"), device="cuda")]
        sfda.sfda_linear_backward(self.q, self.k, self.v, self.log_decay, self.lens, self.S0, self.d_o, self.dS_T, *out, self.scale,
                                  self.workspace(True) if ws == "own" else ws, stream)
        return out

    def arrays(self):
        f = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        n = None if self.lens is None else [min(max(int(x), 0), self.sizes[1]) for x in self.lens]
        return f(self.q), f(self.k), f(self.v), f(self.log_decay), f(self.d_o), f(self.dS_T), n, f(self.S0)

    def oracle(self):
        q, k, v, ld, d_o, dS, n, S0 = self.arrays()
        return op.linear_forward(q, k, v, ld, n, S0, self.scale), op.linear_backward(q, k, v, ld, d_o, dS, n, S0, self.scale)

    def check(self):
        (o, S), (dq, dk, dv, dS0) = self.oracle()
        got_o, got_S = self.forward()
        grads = self.backward()
        torch.cuda.synchronize()
        assert off(got_o, o) <= tol(self.dt) and off(got_S, S) <= tol(self.dt, True), (off(got_o, o), off(got_S, S))
        errors = [off(x, y) for x, y in zip(grads, (dq, dk, dv, dS0))]
        assert max(errors[:3]) <= tol(self.dt) and errors[3] <= tol(self.dt, True), errors


# ---- linear attention: whole sequences -------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 257, 400])
def test_linear_lengths(T, dtype):
    Linear(2, T, 3, dtype=dtype, seed=T).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("T", [40, 150, 300])
def test_linear_widths(T, dk, dv, dtype):
    Linear(1, T, 2, dk=dk, dv=dv, dtype=dtype, seed=5).check()
    Linear(2, T, 2, dk=dk, dv=dv, dtype=dtype, seed=6, state=False).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,H_kv", [(2, 1), (6, 2), (6, 3), (5, 1), (20, 10)])
def test_linear_shared_heads(H, H_kv, dtype):
    Linear(2, 150, H, H_kv, dk=64, dv=128, dtype=dtype, seed=7, lens=[150, 97]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_decays_from_none_to_all(dtype):
    decay = [0.0, -1e-7, -1e-3, -0.05, -0.6, -3.0, -20.0, -120.0, -1e30, -float("inf")]
    Linear(1, 300, len(decay), dtype=dtype, decay=decay, seed=8).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_sequences_of_their_own_length(dtype):
    lens = [0, 1, 64, 65, 127, 128, 129, 200, 199, 1000, -5]
    x = Linear(len(lens), 200, 2, 1, dtype=dtype, lens=lens, seed=9)
    x.check()
    # what lies behind a sequence's end is neither read nor written, not even where it is not finite
    clean = x.forward(fill=7.0) + tuple(x.backward(fill=7.0))
    for b, n in enumerate(lens):
        for t in (x.q, x.k, x.v, x.d_o):
            t[b, max(n, 0):] = float("nan")
    again = x.forward(fill=7.0) + tuple(x.backward(fill=7.0))
    for a, c in zip(clean, again):
        assert torch.equal(a, c)
    for a in clean[0], clean[2], clean[3], clean[4]:
        for b, n in enumerate(lens):
            assert (a[b, max(n, 0):] == 7.0).all()
    assert torch.equal(clean[1][0], x.S0[0]) and torch.equal(clean[5][0], x.dS_T[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_linear_values_that_are_not_finite_reach_only_what_depends_on_them(value, dtype):
    """One such entry of each input by itself; what the formula does not make depend on it has the bits of the clean run."""
    T, t, h, c = 300, 140, 1, 17
    for name in ("q", "k", "v", "d_o"):
        x = Linear(2, T, 3, dtype=dtype, seed=10)
        o, S, dq, dk, dv, dS0 = x.forward() + tuple(x.backward())
        getattr(x, name)[1, t, h, c] = value
        got = x.forward() + tuple(x.backward())
        reach = [torch.zeros_like(y, dtype=torch.bool) for y in got]
        O, ST, DQ, DK, DV, D0 = reach
        if name == "q":
            O[1, t, h] = DQ[0, 0, 0, 0] = True                     # (dq does not depend on q; nothing of it is marked)
            DQ[0, 0, 0, 0] = False
            DK[1, :t + 1, h, c] = True
            DV[1, :t + 1, h] = D0[1, h, c] = True
        elif name == "k":
            O[1, t:, h] = ST[1, h, c] = DQ[1, t:, h, c] = DV[1, t, h] = True
        elif name == "v":
            O[1, t:, h, c] = ST[1, h, :, c] = DQ[1, t:, h] = DK[1, t, h] = True
        else:
            DQ[1, t, h] = DK[1, :t + 1, h] = DV[1, :t + 1, h, c] = D0[1, h, :, c] = True
        for n, (a, clean, r) in enumerate(zip(got, (o, S, dq, dk, dv, dS0), reach)):
            assert torch.equal(a[~r], clean[~r]), (name, n)
            assert not torch.isfinite(a[r]).any(), (name, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_long_sequences_and_few_of_them(dtype):
    Linear(1, 3000, 1, dtype=dtype, decay=[-2.0 ** -10], seed=11).check()
    Linear(1, 2500, 2, 1, dk=64, dv=64, dtype=dtype, decay=[0.0, -2.0 ** -6], seed=12, lens=[2117]).check()


def test_linear_final_state_may_overwrite_the_initial_one():
    for dtype in DTYPES:
        x = Linear(2, 500, 3, dtype=dtype, seed=13)
        o, S = x.forward()
        inplace, o2 = x.S0.clone(), torch.empty_like(o)
        sfda.sfda_linear_forward(x.q, x.k, x.v, x.log_decay, None, inplace, o2, inplace, x.scale, x.workspace())
        assert torch.equal(inplace, S) and torch.equal(o, o2)
        nothing = torch.empty_like(o)
        sfda.sfda_linear_forward(x.q, x.k, x.v, x.log_decay, None, x.S0, nothing, None, x.scale, x.workspace())
        assert torch.equal(nothing, o)


def test_linear_final_state_may_overwrite_the_initial_one_of_cut_sequences():
    """Sequences that are cut into stretches of time, the last of them empty: its CTA writes the final state while others begin."""
    for lens in ([4000], [10], [0], [2100]):
        x = Linear(1, 4000, 2, lens=lens, decay=[-2.0 ** -12, -0.0], seed=44)
        o, S = x.forward()
        (wo, wS), _ = x.oracle()
        assert off(o, wo) <= (BF16 if lens[0] else 0) and off(S, wS) <= STATE
        ws, keep = x.workspace(), x.S0.clone()
        assert ws.numel() > 256 + 4 * S.numel()
        for _ in range(20):
            x.S0.copy_(keep)
            o2 = torch.zeros_like(o)
            sfda.sfda_linear_forward(x.q, x.k, x.v, x.log_decay, x.lens, x.S0, o2, x.S0, x.scale, ws)
            assert torch.equal(x.S0, S) and torch.equal(o2, o)


def test_linear_pieces_of_a_sequence_continue_each_other():
    for dtype in DTYPES:
        x = Linear(1, 700, 2, dtype=dtype, seed=14)
        o, S = x.forward()
        state, parts = x.S0, []
        for a, b in ((0, 1), (1, 130), (130, 386), (386, 700)):
            part, nxt = torch.empty(1, b - a, 2, 128, device="cuda", dtype=x.dt), torch.empty_like(S)
            y = [t[:, a:b].contiguous() for t in (x.q, x.k, x.v)]
            n = sfda.sfda_linear_workspace_bytes(1, b - a, 2, 2, 128, 128, x.code())
            sfda.sfda_linear_forward(*y, x.log_decay, None, state, part, nxt, x.scale, torch.empty(n, device="cuda", dtype=torch.uint8) if n else None)
            parts.append(part)
            state = nxt
        assert off(torch.cat(parts, 1), o.double().cpu().numpy()) <= 2 * tol(x.dt)
        assert off(state, S.double().cpu().numpy()) <= 2 * tol(x.dt, True)


def test_linear_runs_give_the_same_bits_alone_together_and_replayed():
    for dtype in DTYPES:
        for sizes in ((3, 700, 5, 5), (1, 1500, 2, 1)):
            x, y = (Linear(*sizes, dtype=dtype, seed=s) for s in (15, 16))
            want = [z.forward() + tuple(z.backward()) for z in (x, y)]
            torch.cuda.synchronize()
            streams = [torch.cuda.Stream() for _ in range(2)]
            scratch = [(z.workspace(), z.workspace(True)) for z in (x, y)]
            for _ in range(3):
                got = []
                for z, s, ws in zip((x, y), streams, scratch):
                    with torch.cuda.stream(s):
                        got.append(z.forward(ws[0]) + tuple(z.backward(ws[1])))
                torch.cuda.synchronize()
                for a, b in zip(got, want):
                    assert all(torch.equal(i, j) for i, j in zip(a, b))
            ws = scratch[0]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = x.forward(ws[0]) + tuple(x.backward(ws[1]))
            x.q.mul_(2.0)
            fresh = x.forward() + tuple(x.backward())
            for _ in range(2):
                graph.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(i, j) for i, j in zip(got, fresh))


def test_linear_runs_on_the_stream_that_is_named():
    x = Linear(1, 200, 2, seed=17)
    want = x.forward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = x.forward(stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0])


def test_linear_offsets_past_32_bits():
    """q, k, v, o of 2.4e9 elements each: the last sequences have the bits that they have alone."""
    B, T, H = 72, 8192, 32
    x = Linear(B, T, H, state=False, seed=18)
    o, S = x.forward()
    part = Linear(1, 1, 1)
    part.__dict__.update(x.__dict__)
    for b in (0, B - 1):
        part.sizes = (1,) + x.sizes[1:]
        part.q, part.k, part.v = (t[b:b + 1].contiguous() for t in (x.q, x.k, x.v))
        got = part.forward()
        assert off(got[0], o[b:b + 1].double().cpu().numpy()) < BF16 and off(got[1], S[b:b + 1].double().cpu().numpy()) < STATE
    del x, part, o, S
    torch.cuda.empty_cache()


def test_linear_results_do_not_depend_on_the_timing_of_the_roles():
    """The bf16 kernel's roles hand chunks to one another; a development build pauses them at random after arrivals and waits, and
    has to give the same bits: pairs that share a CTA, cut sequences, ends within a chunk, empty ones, both kinds of decays."""
    from paper_2607_11897_b200 import binding
    from paper_2607_11897_b200 import build as cuda_build
    chaos = binding.load_library(cuda_build.build_variant("chaos", ["-DSFDA_WS_CHAOS"]))
    mixed = [-0.001, -0.9, -0.1, -30.0, 0.0, -0.3]
    cases = [Linear(50, 300, 6, decay=mixed, seed=40), Linear(3, 400, 6, 2, decay=mixed, lens=[400, 0, 129], seed=41),
             Linear(1, 4000, 2, decay=[-0.01, -2.0], seed=42), Linear(40, 130, 6, dk=64, dv=128, decay=mixed, lens=[1, 130, 0, 128] * 10, seed=43)]
    for x in cases:
        want = x.forward() + tuple(x.backward())
        plain, ws = binding.load(), x.workspace()
        binding._LIB = chaos
        try:
            for _ in range(3):
                got = x.forward(ws) + tuple(x.backward())
                assert all(torch.equal(a, b) for a, b in zip(got, want))
                assert sfda.sfda_workspace_status(ws) == 0
        finally:
            binding._LIB = plain


# ---- linear attention: one token -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("B,H,H_kv", [(1, 1, 1), (3, 4, 2), (40, 6, 6)])
def test_linear_steps_are_the_recurrence(B, H, H_kv, dk, dv, dtype):
    x = Linear(B, 5, H, H_kv, dk=dk, dv=dv, dtype=dtype, seed=19, decay=([0.0, -0.3, -float("inf"), -2.0, -1e-6, -40.0] * H)[:H])
    (o, S_T), _ = x.oracle()
    S, rows = x.S0.clone(), []
    for t in range(5):
        out = torch.empty(B, H, dv, device="cuda", dtype=x.dt)
        sfda.sfda_linear_step(x.q[:, t].contiguous(), x.k[:, t].contiguous(), x.v[:, t].contiguous(), x.log_decay, S, out, x.scale)
        rows.append(out)
    assert off(S, S_T) <= 1e-6                                   # five fp32 updates: 10 roundings of 2^-24
    assert off(torch.stack(rows, 1), o) <= (2e-6 if dtype == "f32" else ROUND)


def test_linear_steps_of_a_slow_decay_do_not_drift():
    """4096 decays by 1 - 2^-14 without input: each multiplication rounds by 2^-24 in a random direction, sqrt(4096) of them in
    all; a factor whose own rounding (up to 2^-25) came back every time would be off by 4096 of those, 1.2e-4."""
    S = torch.randn(1, 1, 128, 128, device="cuda")
    want = S.double() * np.exp(4096 * float(np.float32(-(2.0 ** -14))))
    z, out = torch.zeros(1, 1, 128, device="cuda"), torch.empty(1, 1, 128, device="cuda")
    ld = torch.tensor([-(2.0 ** -14)], device="cuda")
    for _ in range(4096):
        sfda.sfda_linear_step(z, z, z, ld, S, out)
    assert off(S, want.cpu().numpy()) < 1e-5


def test_linear_step_can_be_captured():
    x = Linear(4, 1, 8, 4, seed=20)
    q, k, v = (t[:, 0].contiguous() for t in (x.q, x.k, x.v))
    out, S = torch.empty(4, 8, 128, device="cuda", dtype=x.dt), x.S0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            sfda.sfda_linear_step(q, k, v, x.log_decay, S, out, x.scale)
    S.copy_(x.S0)
    graph.replay()
    want, out2 = x.S0.clone(), torch.empty_like(out)
    for _ in range(3):
        sfda.sfda_linear_step(q, k, v, x.log_decay, want, out2, x.scale)
    torch.cuda.synchronize()
    assert torch.equal(S, want) and torch.equal(out, out2)


# ---- rotary positions ------------------------------------------------------------------------------------------------
def rotary_case(B, T, H, H_kv, d, rot, dtype, far=1000, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, T, H, d, device="cuda", generator=g).to(DTYPES[dtype])
    k = torch.randn(B, T, H_kv, d, device="cuda", generator=g).to(DTYPES[dtype])
    pos = torch.randint(-far, far + 1, (B, T), device="cuda", generator=g, dtype=torch.int32)
    return q, k, pos, sfda.sfda_rotary_turns(rot).cuda() if rot else torch.empty(0, dtype=torch.int64, device="cuda")


def check_rotary(q, k, pos, turns, halves, amplitude, inverse, got):
    f = op.rotary_frequencies(2 * turns.numel())
    for x, y in ((q, got[0]), (k, got[1])):
        want = op.rotary(x.double().cpu().numpy(), pos.cpu().numpy(), f, halves, amplitude, inverse)
        # fp32: the angle to 2^-25 of half a turn, sines to 2 ulp, three operations: under 8 * 2^-24.  The oracle's own angle,
        # position times frequency in doubles, is 2^-53 of itself off.
        assert off(y, want) <= (5e-7 if x.dtype == torch.float32 else ROUND)
        keep = 2 * turns.numel()
        assert torch.equal(y[..., keep:], x[..., keep:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 32), (128, 126), (96, 24), (96, 90), (80, 40), (256, 254), (2, 2), (6, 4), (10, 0), (64, 2), (1024, 512)])
def test_rotary_layouts_and_widths(d, rot, halves, dtype):
    q, k, pos, turns = rotary_case(2, 7, 3, 1, d, rot, dtype, seed=d + rot)
    if not rot:
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        rc = sfda.load().sfda_rotary(q.data_ptr(), k.data_ptr(), pos.data_ptr(), None, q_out.data_ptr(), k_out.data_ptr(), 2, 7, 3, 1,
                                     d, 0, 3 * d, d, 3 * d, d, int(halves), 1.0, 0, int(dtype == "bf16"), None)
        torch.cuda.synchronize()
        assert rc == 0 and torch.equal(q_out, q) and torch.equal(k_out, k)
        return
    for inverse in (False, True):
        got = torch.empty_like(q), torch.empty_like(k)
        sfda.sfda_rotary(q, k, pos, turns, *got, int(halves), 1.25, inverse)
        check_rotary(q, k, pos, turns, halves, 1.25, inverse, got)


@pytest.mark.parametrize("B,T,H,H_kv", [(1, 1, 1, 1), (3, 1, 33, 7), (1, 513, 8, 8), (2, 100, 9, 1), (1, 4099, 2, 2)])
def test_rotary_numbers_of_tokens_and_heads(B, T, H, H_kv):
    for halves in (False, True):
        q, k, pos, turns = rotary_case(B, T, H, H_kv, 64, 64, "bf16", seed=3)
        got = torch.empty_like(q), torch.empty_like(k)
        sfda.sfda_rotary(q, k, pos, turns, *got, int(halves))
        check_rotary(q, k, pos, turns, halves, 1.0, False, got)


def test_rotary_far_positions_are_exact():
    """At the end of int32 an angle in fp32 would be off by whole turns; counts modulo 2^64 are not."""
    q, k, _, turns = rotary_case(1, 6, 2, 2, 64, 64, "f32")
    pos = torch.tensor([[0, 1 << 20, 123456789, 2 ** 31 - 1, -(2 ** 31), -77777777]], device="cuda", dtype=torch.int32)
    # the fastest pair's oracle angle, 2^31 radians in doubles, is good to 2^-22; the others are slower
    for halves in (0, 1):
        got = torch.empty_like(q), torch.empty_like(k)
        sfda.sfda_rotary(q, k, pos, turns, *got, halves)
        want = op.rotary(q.double().cpu().numpy(), pos.cpu().numpy(), op.rotary_frequencies(64), bool(halves))
        assert off(got[0], want) <= 5e-7 + 2.0 ** -22


def test_rotary_slices_of_a_packed_projection_in_place_and_alone():
    B, T, H, H_kv, d = 2, 37, 4, 2, 64
    for dtype in DTYPES:
        for halves in (0, 1):
            packed = torch.randn(B, T, (H + 2 * H_kv) * d, device="cuda").to(DTYPES[dtype])
            q = packed[..., :H * d].unflatten(-1, (H, d))
            k = packed[..., H * d:(H + H_kv) * d].unflatten(-1, (H_kv, d))
            pos = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1)
            turns = sfda.sfda_rotary_turns(48).cuda()
            dense = torch.empty(B, T, H, d, device="cuda", dtype=q.dtype), torch.empty(B, T, H_kv, d, device="cuda", dtype=q.dtype)
            sfda.sfda_rotary(q, k, pos, turns, *dense, halves)
            check_rotary(q, k, pos, turns, bool(halves), 1.0, False, dense)
            before = packed.clone()
            sfda.sfda_rotary(q, k, pos, turns, q, k, halves)
            assert torch.equal(q, dense[0]) and torch.equal(k, dense[1])
            assert torch.equal(packed[..., (H + H_kv) * d:], before[..., (H + H_kv) * d:])
            alone = torch.empty_like(dense[0])
            sfda.sfda_rotary(before[..., :H * d].unflatten(-1, (H, d)), None, pos, turns, alone, None, halves)
            assert torch.equal(alone, dense[0])
            # one token per sequence, and a stride that no wide access divides
            odd = torch.randn(5, H * d + 2, device="cuda").to(q.dtype)
            step = odd[:, :H * d].unflatten(-1, (H, d))
            out = torch.empty(5, H, d, device="cuda", dtype=q.dtype)
            sfda.sfda_rotary(step, None, pos[0, 20:25].contiguous(), turns, out, None, halves)
            want = op.rotary(step.double().cpu().numpy()[:, None], pos[0, 20:25, None].cpu().numpy(), op.rotary_frequencies(48), bool(halves))
            assert off(out, want[:, 0]) <= (5e-7 if dtype == "f32" else ROUND)


def test_rotary_copies_what_it_does_not_turn_bit_for_bit():
    q, k, pos, turns = rotary_case(1, 3, 2, 1, 64, 20, "bf16")
    q[..., 20:] = torch.tensor([float("nan"), float("inf"), -0.0, 1.0], device="cuda").repeat(11)
    for halves in (0, 1):
        got = torch.empty_like(q), torch.empty_like(k)
        sfda.sfda_rotary(q, k, pos, turns, *got, halves)
        assert torch.equal(got[0][..., 20:].view(torch.int16), q[..., 20:].view(torch.int16))
        assert torch.isfinite(got[0][..., :20]).all()


def test_rotary_refuses_other_layouts():
    q, k, pos, turns = rotary_case(2, 4, 2, 2, 64, 64, "bf16")
    with pytest.raises(ValueError):
        sfda.sfda_rotary(q.transpose(2, 3), k, pos, turns, q, k)
    with pytest.raises(ValueError):
        sfda.sfda_rotary(q, k, pos[:, :3].contiguous(), turns, q, k)
    with pytest.raises(ValueError):
        sfda.sfda_rotary(q, k, pos, turns, torch.empty(2, 4, 3, 64, device="cuda", dtype=q.dtype), k)
    with pytest.raises(TypeError):
        sfda.sfda_rotary(q, k.float(), pos, turns, q, k)
    with pytest.raises(ValueError):                              # two strides that are not one
        x = torch.empty(2, 6, 2, 64, device="cuda", dtype=q.dtype)[:, :4]
        sfda.sfda_rotary(x, None, pos, turns, q, None)


# ---- group norm ------------------------------------------------------------------------------------------------------
def norm_case(rows, C, dtype, gated, affine, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, gate, dy = ((r(rows, C) * 2 + r(1, C)).to(DTYPES[dtype]), r(rows, C).to(DTYPES[dtype]) if gated else None, r(rows, C).to(DTYPES[dtype]))
    return x, r(C) if affine else None, r(C) if affine else None, gate, dy


def check_norm(rows, C, groups, dtype, act, gated, affine, eps=1e-5, seed=0):
    x, w, b, gate, dy = norm_case(rows, C, dtype, gated, affine, seed)
    f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    y = torch.empty_like(x)
    sfda.sfda_group_norm(x, w, b, gate, y, groups, eps, act)
    dx, dgate = torch.empty_like(x), torch.empty_like(x) if gated else None
    dw, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(sfda.sfda_group_norm_backward_workspace_bytes(rows, C), device="cuda", dtype=torch.uint8)
    sfda.sfda_group_norm_backward(x, w, b, gate, dy, dx, dw, db, dgate, groups, eps, act, ws)
    want = op.group_norm(f(x), f(w), f(b), f(gate), groups, eps, act == sfda.SFDA_ACT_SILU)
    gx, gw, gb, gg = op.group_norm_backward(f(x), f(w), f(b), f(gate), f(dy), groups, eps, act == sfda.SFDA_ACT_SILU)
    # fp32: mean and variance of a few hundred terms, a dozen operations: 2e-6; one rounding of half a step for bf16
    t = 2e-6 if dtype == "f32" else ROUND
    got = dict(y=off(y, want), dx=off(dx, gx), dw=off(dw, gw) / 4, db=off(db, gb) / 4)
    if gated:
        got["dgate"] = off(dgate, gg)
    assert all(v <= (2e-6 if n in ("dw", "db") else t) for n, v in got.items()), got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,C,groups", [(1, 64, 1), (5, 4096, 32), (300, 2560, 20), (17, 96, 1), (33, 7 * 36, 7), (9, 500, 5), (3, 30, 2)])
def test_group_norm_shapes(rows, C, groups, gated, act, dtype):
    check_norm(rows, C, groups, dtype, act, gated, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C,groups", [(4, 512, 1), (3, 1024, 1), (2, 2048, 2), (5, 8192, 1), (3, 5003, 1), (2, 127 * 3, 3), (2, 129 * 3, 3), (70, 3, 3 // 3)])
def test_group_norm_wide_and_odd_groups(rows, C, groups, dtype):
    check_norm(rows, C, groups, dtype, 1, True, True)
    check_norm(rows, C, groups, dtype, 1, False, False)


@pytest.mark.parametrize("rows", [2, 1183, 1185, 20000])
def test_group_norm_numbers_of_rows(rows):
    check_norm(rows, 128, 2, "bf16", 1, True, True, seed=rows)
    check_norm(rows, 40, 1, "f32", 0, False, True, seed=rows)


def test_group_norm_of_constant_rows_is_the_bias():
    x = torch.full((4, 256), 3.0, device="cuda")
    w, b, y = torch.randn(256, device="cuda"), torch.randn(256, device="cuda"), torch.empty(4, 256, device="cuda")
    sfda.sfda_group_norm(x, w, b, None, y, 2)
    assert torch.equal(y, b.expand(4, 256))


def test_group_norm_keeps_small_variances_about_a_large_mean():
    """Differences of 1 about 4096 in fp32: sums of squares would keep 2^-24 of 4096^2 = 1, all of the variance."""
    x = 4096.0 + torch.randn(8, 128, device="cuda").double()
    x = x.float()
    y = torch.empty_like(x)
    sfda.sfda_group_norm(x, None, None, None, y, 1)
    # the mean is rounded to 2^-24 of 4096, 2.4e-4 of the unit deviation, and so is every difference taken from it
    assert off(y, op.group_norm(x.double().cpu().numpy(), None, None, None, 1, 1e-5, False)) < 5e-4


def test_group_norm_writes_over_its_input_and_keeps_rows_apart():
    x, w, b, gate, dy = norm_case(50, 256, "bf16", True, True)
    y = torch.empty_like(x)
    sfda.sfda_group_norm(x, w, b, gate, y, 4, 1e-5, 1)
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    sfda.sfda_group_norm_backward(x, w, b, gate, dy, dx, None, None, dg, 4, 1e-5, 1)
    for over in (x, gate):
        a, g = x.clone(), gate.clone()
        sfda.sfda_group_norm(a, w, b, g, a if over is x else g, 4, 1e-5, 1)
        assert torch.equal(a if over is x else g, y)
    d, g = dy.clone(), gate.clone()
    sfda.sfda_group_norm_backward(x, w, b, g, d, d, None, None, g, 4, 1e-5, 1)
    assert torch.equal(d, dx) and torch.equal(g, dg)
    x[7, 3] = float("nan")
    z = torch.empty_like(x)
    sfda.sfda_group_norm(x, w, b, gate, z, 4, 1e-5, 1)
    bad = torch.zeros_like(z, dtype=torch.bool)
    bad[7, :64] = True
    assert torch.equal(z[~bad], y[~bad]) and torch.isnan(z[bad]).all()


@pytest.mark.parametrize("C,groups", [(16384, 1), (5003, 1), (4096, 1), (3 * 1500, 3), (144, 4)])
def test_group_norm_gradients_may_lie_over_their_inputs(C, groups):
    x, w, b, gate, dy = norm_case(6, C, "bf16", True, True)
    ws = torch.empty(sfda.sfda_group_norm_backward_workspace_bytes(6, C), device="cuda", dtype=torch.uint8)
    want = [torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), torch.empty_like(x)]
    sfda.sfda_group_norm_backward(x, w, b, gate, dy, *want, groups, 1e-5, 1, ws)
    dw, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    sfda.sfda_group_norm_backward(x, w, b, gate, dy, dy, dw, db, gate, groups, 1e-5, 1, ws)
    assert all(torch.equal(i, j) for i, j in zip((dy, dw, db, gate), want))


def test_operators_run_on_the_stream_that_is_named():
    """Each on a stream of its own while the default one is busy: what it reads is written on that stream, right before."""
    s = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    x, w, b, gate, dy = norm_case(64, 256, "bf16", True, True)
    q, k, pos, turns = rotary_case(2, 9, 4, 2, 64, 64, "bf16")
    step = Linear(2, 1, 4, dk=64, dv=64, seed=45)
    args = [t[:, 0].contiguous() for t in (step.q, step.k, step.v)]
    results = []
    for stream in (None, s):
        y, q2, k2, S, o = torch.empty_like(x), torch.empty_like(q), torch.empty_like(k), step.S0.clone(), torch.empty(2, 4, 64, device="cuda", dtype=step.dt)
        torch.cuda.synchronize()
        if stream is not None:
            for _ in range(5):
                big = (big @ big).clamp_(-1, 1)
        with torch.cuda.stream(stream):
            x2, qq = x * 2, q * 2
        sfda.sfda_group_norm(x2, w, b, gate, y, 4, 1e-5, 1, stream)
        sfda.sfda_rotary(qq, k, pos, turns, q2, k2, 0, 1.0, False, stream)
        sfda.sfda_linear_step(*args, step.log_decay, S, o, 1.0, stream)
        torch.cuda.synchronize()
        results.append((y, q2, k2, S, o))
    assert all(torch.equal(i, j) for i, j in zip(*results))


def test_group_norm_sums_are_the_same_bits_every_time_and_captured():
    x, w, b, gate, dy = norm_case(5000, 512, "bf16", True, True)
    ws = torch.empty(sfda.sfda_group_norm_backward_workspace_bytes(5000, 512), device="cuda", dtype=torch.uint8)

    def run():
        out = [torch.empty_like(x), torch.empty(512, device="cuda"), torch.empty(512, device="cuda"), torch.empty_like(x)]
        sfda.sfda_group_norm_backward(x, w, b, gate, dy, *out, 4, 1e-5, 1, ws)
        return out
    first = run()
    for _ in range(3):
        assert all(torch.equal(i, j) for i, j in zip(first, run()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(i, j) for i, j in zip(first, got))


# ---- a layer ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_of_the_three_and_its_gradients(dtype):
    """Rotation, attention, norm with a gate, as one layer uses them, and back; then its tokens one at a time."""
    B, T, H, H_kv, d, dt = 2, 150, 4, 2, 64, DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(30)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, gate, dy = (r(B, T, n, d).to(dt) for n in (H, H_kv, H_kv, H, H))
    w, b, ld = 1 + 0.1 * r(H * d), 0.1 * r(H * d), -0.1 * torch.rand(H, device="cuda", generator=g)
    pos = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1)
    turns, scale = sfda.sfda_rotary_turns(d).cuda(), d ** -0.5
    e = torch.empty_like
    qr, kr, o, y = e(q), e(k), e(q), e(q)
    S = torch.empty(B, H, d, d, device="cuda")
    code = sfda.SFDA_BF16 if dtype == "bf16" else sfda.SFDA_F32
    scratch = lambda n: torch.empty(n, device="cuda", dtype=torch.uint8) if n else None  # noqa: E731
    sfda.sfda_rotary(q, k, pos, turns, qr, kr)
    sfda.sfda_linear_forward(qr, kr, v, ld, None, None, o, S, scale, scratch(sfda.sfda_linear_workspace_bytes(B, T, H, H_kv, d, d, code)))
    flat = lambda t: t.view(B * T, H * d)  # noqa: E731
    sfda.sfda_group_norm(flat(o), w, b, flat(gate), flat(y), H, 1e-5, 1)
    do, dgate, dw, db = e(o), e(gate), torch.empty(H * d, device="cuda"), torch.empty(H * d, device="cuda")
    sfda.sfda_group_norm_backward(flat(o), w, b, flat(gate), flat(dy), flat(do), dw, db, flat(dgate), H, 1e-5, 1,
                                  scratch(sfda.sfda_group_norm_backward_workspace_bytes(B * T, H * d)))
    dq, dk, dv, dS0 = e(q), e(k), e(v), e(S)
    sfda.sfda_linear_backward(qr, kr, v, ld, None, None, do, None, dq, dk, dv, dS0, scale,
                              scratch(sfda.sfda_linear_backward_workspace_bytes(B, T, H, H_kv, d, d, code)))
    sfda.sfda_rotary(dq, dk, pos, turns, dq, dk, inverse=True)

    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    n = lambda t: f(t).reshape(B * T, H * d)  # noqa: E731
    fr = op.rotary_frequencies(d)
    Q, K = op.rotary(f(q), f(pos), fr), op.rotary(f(k), f(pos), fr)
    O, ST = op.linear_forward(Q, K, f(v), f(ld), scale=scale)
    Y = op.group_norm(O.reshape(B * T, H * d), f(w), f(b), n(gate), H, 1e-5, True)
    dO, dW, dB, dG = op.group_norm_backward(O.reshape(B * T, H * d), f(w), f(b), n(gate), n(dy), H, 1e-5, True)
    gq, gk, gv, _ = op.linear_backward(Q, K, f(v), f(ld), dO.reshape(O.shape), scale=scale)
    gq, gk = op.rotary(gq, f(pos), fr, inverse=True), op.rotary(gk, f(pos), fr, inverse=True)
    # in bf16 the operators hand rounded tensors to each other: up to ten roundings on the longest way (q, k turned; scores,
    # state, o; d_o; scores, state, dq; dq turned), each (eps / 2) / sqrt(3), amplified at most twice by the norm's derivative
    t = 20 * F32 if dtype == "f32" else 20 * ROUND / 3 ** 0.5
    got = dict(y=off(flat(y), Y), S=off(S, ST), dgate=off(flat(dgate), dG), dw=off(dw, dW), db=off(db, dB), dq=off(dq, gq), dk=off(dk, gk), dv=off(dv, gv))
    assert max(got.values()) <= t, got

    state, worst = torch.zeros_like(S), 0.0
    for i in range(T):
        qt, kt, vt = (x[:, i].contiguous() for x in (q, k, v))
        ot, yt = torch.empty_like(qt), torch.empty_like(qt)
        sfda.sfda_rotary(qt, kt, pos[:, i].contiguous(), turns, qt, kt)
        sfda.sfda_linear_step(qt, kt, vt, ld, state, ot, scale)
        sfda.sfda_group_norm(ot.view(B, H * d), w, b, gate[:, i].contiguous().view(B, H * d), yt.view(B, H * d), H, 1e-5, 1)
        worst = max(worst, off(yt.view(B, H * d), Y.reshape(B, T, H * d)[:, i]))
    assert worst <= t, worst
