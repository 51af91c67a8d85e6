"""Test infrastructure: the operators around linear attention with a fixed decay for each head, in float64, each from its
definition (token by token, pair by pair, group by group).  Shares no code with the CUDA path."""
import numpy as np


def _spread(x, H):
    """[B, T, H_kv, d] -> [B, T, H, d]: every key and value head under the query heads that read it."""
    return np.repeat(np.asarray(x, np.float64), H // x.shape[2], axis=2)


def linear_forward(q, k, v, log_decay, lens=None, S0=None, scale=1.0):
    """S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t.  Returns (o, S_T); rows behind a sequence's end are 0."""
    B, T, H, dk = q.shape
    q, k, v = np.asarray(q, np.float64), _spread(k, H), _spread(v, H)
    gamma = np.exp(np.asarray(log_decay, np.float64))
    o = np.zeros((B, T, H, v.shape[3]))
    S = np.zeros((B, H, dk, v.shape[3])) if S0 is None else np.array(S0, np.float64)
    for b in range(B):
        for t in range(T if lens is None else int(lens[b])):
            S[b] = gamma[:, None, None] * S[b] + k[b, t, :, :, None] * v[b, t, :, None, :]
            o[b, t] = scale * np.einsum("hk,hkv->hv", q[b, t], S[b])
    return o, S


def linear_backward(q, k, v, log_decay, d_o, dS_T=None, lens=None, S0=None, scale=1.0):
    """Gradients of sum(d_o o) + sum(dS_T S_T): (dq, dk, dv, dS0), those of shared heads summed."""
    B, T, H, dk = q.shape
    H_kv, dv = v.shape[2:]
    q, k, v, d_o = np.asarray(q, np.float64), _spread(k, H), _spread(v, H), np.asarray(d_o, np.float64)
    gamma = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    gq, gk, gv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    G0 = np.zeros((B, H, dk, dv)) if dS_T is None else np.array(dS_T, np.float64)
    for b in range(B):
        n = T if lens is None else int(lens[b])
        S = np.zeros((H, dk, dv)) if S0 is None else np.array(S0[b], np.float64)
        for t in range(n):
            S = gamma * S + k[b, t, :, :, None] * v[b, t, :, None, :]
            gq[b, t] = scale * np.einsum("hkv,hv->hk", S, d_o[b, t])
        for t in reversed(range(n)):
            G = G0[b] + scale * q[b, t, :, :, None] * d_o[b, t, :, None, :]
            gk[b, t] = np.einsum("hkv,hv->hk", G, v[b, t])
            gv[b, t] = np.einsum("hkv,hk->hv", G, k[b, t])
            G0[b] = gamma * G
    share = lambda x: x.reshape(B, T, H_kv, H // H_kv, -1).sum(3)  # noqa: E731
    return gq, share(gk), share(gv), G0


def rotary_frequencies(rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=4.0, trained=8192.0):
    """Radians per position of every pair."""
    out = []
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "base" else base
        f = b ** (-2.0 * j / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            s = min(1.0, max(0.0, (trained * f / (2 * np.pi) - low) / (high - low)))
            f = s * f + (1 - s) * f / factor
        out.append(f)
    return np.array(out)


def rotary(x, positions, frequencies, halves=False, amplitude=1.0, inverse=False):
    """x [B, T, heads, d]: each pair of the first 2 len(frequencies) channels times amplitude e^(+-i position frequency)."""
    y, half = np.array(x, np.float64), len(frequencies)
    angle = np.asarray(positions, np.float64)[..., None] * frequencies * (-1.0 if inverse else 1.0)
    turn = (amplitude * np.exp(1j * angle))[:, :, None, :]
    for j in range(half):
        re, im = (j, j + half) if halves else (2 * j, 2 * j + 1)
        z = (np.asarray(x, np.float64)[..., re] + 1j * np.asarray(x, np.float64)[..., im]) * turn[..., j]
        y[..., re], y[..., im] = z.real, z.imag
    return y


def _silu(u):
    s = 1.0 / (1.0 + np.exp(-u))
    return u * s, s * (1.0 + u * (1.0 - s))


def group_norm(x, weight, bias, gate, groups, eps, silu):
    """y of x [rows, C]: (x - mean) / sqrt(var + eps) over each group, affine, then act(z) or z act(gate)."""
    return _group_norm(x, weight, bias, gate, groups, eps, silu)[0]


def _group_norm(x, weight, bias, gate, groups, eps, silu):
    x = np.asarray(x, np.float64)
    rows, C = x.shape
    g = x.reshape(rows, groups, C // groups)
    rstd = 1.0 / np.sqrt(g.var(-1, keepdims=True) + eps)
    n = ((g - g.mean(-1, keepdims=True)) * rstd).reshape(rows, C)
    z = n * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    u = z if gate is None else np.asarray(gate, np.float64)
    a, slope = _silu(u) if silu else (u, np.ones_like(u))
    return (a if gate is None else z * a), n, z, a, slope, rstd


def group_norm_backward(x, weight, bias, gate, dy, groups, eps, silu):
    """(dx, dweight, dbias, dgate) of sum(dy y)."""
    _, n, z, a, slope, rstd = _group_norm(x, weight, bias, gate, groups, eps, silu)
    dy = np.asarray(dy, np.float64)
    rows, C = n.shape
    dz = dy * (slope if gate is None else a)
    dn = (dz * (1.0 if weight is None else np.asarray(weight, np.float64))).reshape(rows, groups, -1)
    ng = n.reshape(rows, groups, -1)
    dx = rstd * (dn - dn.mean(-1, keepdims=True) - ng * (dn * ng).mean(-1, keepdims=True))
    return dx.reshape(rows, C), (dz * n).sum(0), dz.sum(0), None if gate is None else dy * z * slope
