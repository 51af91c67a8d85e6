"""Calls of the operators beside the recurrence that their documentation allows and that are easy to get wrong: inputs that share an
address, parameters that are not finite, groups of one value, named streams."""
import pytest
import torch

import paper_2607_11897_b200 as sfda

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
