"""The operators of a linear-attention layer with a fixed decay for every head, beside the recurrence with rotations and
erasure: the attention itself (whole sequences, their gradients, one token at a time), the rotation of queries and keys
by position before it, and the normalisation of every head's output after it.

A case is a dict of plain values.  Its "kind" is one of

  "step"        one token for B * H states                                                     (sfda_linear_step)
  "prefill"     the chunkwise forward of whole sequences                                       (sfda_linear_forward)
  "train"       the forward and the gradients of a loss on it           (sfda_linear_forward, sfda_linear_backward)
  "rotary"      queries and keys turned by their positions, or gradients turned back                  (sfda_rotary)
  "norm"        group norm over each head's channels, affine, activated or gated                  (sfda_group_norm)
  "norm_train"  the same and its gradients                              (sfda_group_norm, sfda_group_norm_backward)

and the rest are sizes, types ("bf16" or "f32") and switches.

The attention:   S_t = gamma_h S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   gamma_h = exp(log_decay[h]) in (0, 1).
Keys and values may have fewer heads than queries and decays: query head h reads head h // (H / H_kv).  `lens` gives
every sequence its own number of tokens; rows behind it are not written.

Keys are of unit length, q and v ~ N(0, 1), initial states ~ N(0, 0.02); the heads' decays remember between 2 and 4096
tokens, spread over their logarithm.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
C = 64          # chunk of the plain form
TURN = 2.0 * math.pi


def _linear(kind, B, T, H, H_kv, d_k, d_v, dtype, state=False, ragged=False, name=None):
    c = dict(kind=kind, B=B, T=T, H=H, H_kv=H_kv, d_k=d_k, d_v=d_v, dtype=dtype, state=state, ragged=ragged)
    if name is not None:
        c["name"] = name
    return c


def _rotary(B, T, H, H_kv, d, rot, dtype, layout, scaled=False, inverse=False, far=0, name=None):
    c = dict(kind="rotary", B=B, T=T, H=H, H_kv=H_kv, d=d, rot=rot, dtype=dtype, layout=layout, scaled=scaled, inverse=inverse,
             far=far)
    if name is not None:
        c["name"] = name
    return c


def _norm(kind, rows, groups, width, dtype, act="silu", gate=True, affine=True, name=None):
    c = dict(kind=kind, rows=rows, groups=groups, width=width, dtype=dtype, act=act, gate=gate, affine=affine)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one conversation decoding token by token: latency
        _linear("step", 1, 1, 32, 32, 128, 128, "bf16", name="step_one_sequence"),
        # a full serving batch: the states go through memory once
        _linear("step", 256, 1, 32, 32, 128, 128, "bf16", name="step_batch_256"),
        # the small fp32 configuration: unit tests, debugging, toy models
        _linear("prefill", 1, 256, 2, 2, 64, 64, "f32", name="prefill_tiny_fp32"),
        # a batch of prompts padded to the longest one, keys and values shared by two query heads, state carried over
        _linear("prefill", 16, 575, 20, 10, 128, 128, "bf16", state=True, ragged=True, name="prefill_ragged_shared"),
        # large-batch prefill
        _linear("prefill", 8, 8192, 32, 32, 128, 128, "bf16", state=True, name="prefill_headline"),
        # few sequences of 131072 tokens
        _linear("prefill", 1, 131072, 16, 16, 128, 128, "bf16", name="prefill_long"),
        # one training step of a layer, 4096 tokens
        _linear("train", 4, 4096, 16, 16, 128, 128, "bf16", name="train_4k"),
        # fine-tuning a small fp32 model on sequences of odd length, state carried between segments
        _linear("train", 2, 333, 4, 4, 64, 64, "f32", state=True, name="train_small_fp32"),
        # the token of every sequence in a serving batch, somewhere in a long context: latency
        _rotary(256, 1, 32, 8, 128, 128, "bf16", "halves", scaled=True, far=1 << 20, name="rotary_step_far"),
        # queries and keys of a large prefill batch, adjacent channels paired
        _rotary(8, 8192, 32, 32, 128, 128, "bf16", "pairs", name="rotary_prefill"),
        # the outputs of one token per sequence, gated
        _norm("norm", 256, 32, 128, "bf16", name="norm_step_gated"),
        # the outputs of a training batch, gated, and all gradients
        _norm("norm_train", 65536, 32, 128, "bf16", name="norm_train"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["step", "prefill", "prefill", "prefill", "train", "train", "rotary", "rotary", "norm", "norm_train"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H = rng.choice([1, 2, 4, 6, 8, 12, 16, 20, 24, 32])
    H_kv = H if rng.random() < 0.7 else rng.choice([h for h in range(1, H + 1) if H % h == 0])
    if kind in ("step", "prefill", "train"):
        d_k, d_v = (128, 128) if rng.random() < 0.6 else (rng.choice([64, 128]), rng.choice([64, 128]))
        if kind == "step":
            return _linear(kind, _log_uniform(rng, 1, 256), 1, H, H_kv, d_k, d_v, dtype)
        # tokens times heads from 128 to the kind's largest; one token to the longest sequence, round or not
        most = {("prefill", "bf16"): 1 << 21, ("prefill", "f32"): 1 << 18, ("train", "bf16"): 1 << 19, ("train", "f32"): 1 << 17}
        rows = _log_uniform(rng, 128, most[kind, dtype])
        T = _log_uniform(rng, 1, min(131072, max(1, rows // H)))
        if rng.random() < 0.3:
            T = max(1, T // 128 * 128)
        B = max(1, min(64, rows // (T * H)))
        return _linear(kind, B, T, H, H_kv, d_k, d_v, dtype, state=rng.random() < 0.5, ragged=rng.random() < 0.4)
    if kind == "rotary":
        d = rng.choice([64, 64, 96, 128, 128, 128, 192, 256])
        rot = d if rng.random() < 0.6 else rng.choice([d // 4, d // 2, d - 2])
        rows = _log_uniform(rng, 1, (1 << 27) // (H * d))
        T = 1 if rng.random() < 0.25 else _log_uniform(rng, 1, min(rows, 131072))
        B = max(1, min(256, rows // T))
        return _rotary(B, T, H, H_kv, d, rot // 2 * 2, dtype, rng.choice(["pairs", "halves"]), scaled=rng.random() < 0.5,
                       inverse=rng.random() < 0.3, far=rng.choice([0, 0, 4096, 1 << 17, 1 << 20]))
    width = rng.choice([64, 64, 128, 128, 128, 256, 512, 96, 36, 100])
    groups = rng.choice([1, 2, 4, 8, 16, 20, 32])
    rows = _log_uniform(rng, 1, (1 << 26) // (groups * width))
    return _norm(kind, rows, groups, width, dtype, act=rng.choice(["none", "silu"]), gate=rng.random() < 0.6,
                 affine=rng.random() < 0.8)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, std=1.0):
        x = torch.randn(*shape, device="cuda", generator=self.g)
        return x if std == 1.0 else x.mul_(std)

    def uniform(self, lo, hi, *shape):
        return torch.rand(*shape, device="cuda", generator=self.g).mul_(hi - lo).add_(lo)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _unit(x):
    return x.div_(x.norm(dim=-1, keepdim=True))


def _frequencies(case):
    """Radians per token of every rotated pair; a scaled table slows the pairs whose wavelength passes the trained context."""
    f = 10000.0 ** (-np.arange(0, case["rot"], 2, dtype=np.float64) / case["rot"])
    if case["scaled"]:
        factor, low, high, trained = 8.0, 1.0, 4.0, 8192.0
        share = np.clip((trained * f / TURN - low) / (high - low), 0.0, 1.0)
        f = share * f + (1.0 - share) * f / factor
    return f


def prepare(case, seed):
    r, dt, kind = _Draw(seed), _dtype(case), case["kind"]
    s = dict(case=dict(case))
    zeros = lambda *shape, dtype=torch.float32: torch.zeros(*shape, device="cuda", dtype=dtype)  # noqa: E731
    if kind == "rotary":
        B, T, H, H_kv, d = (case[x] for x in ("B", "T", "H", "H_kv", "d"))
        s["q"], s["k"] = r.normal(B, T, H, d).to(dt), r.normal(B, T, H_kv, d).to(dt)
        start = (r.uniform(0, 1, B, 1) * (case["far"] + 1)).to(torch.int32)
        s["positions"] = (start + torch.arange(T, device="cuda", dtype=torch.int32)).contiguous()
        # the table that a program keeps: 2^64 counts to the turn, so that position times frequency wraps by itself
        turns = np.rint(_frequencies(case) / TURN * 2.0 ** 64).astype(np.uint64).view(np.int64)
        s["turns"] = torch.from_numpy(turns).cuda()
        s["amplitude"] = 0.1 * math.log(8.0) + 1.0 if case["scaled"] else 1.0
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s
    if kind in ("norm", "norm_train"):
        rows, channels = case["rows"], case["groups"] * case["width"]
        s["x"] = r.normal(rows, channels).mul_(torch.exp(r.normal(rows, 1))).add_(r.normal(1, channels, std=0.5)).to(dt)
        s["gate"] = r.normal(rows, channels).to(dt) if case["gate"] else None
        s["weight"] = r.normal(channels, std=0.1).add_(1.0) if case["affine"] else None
        s["bias"] = r.normal(channels, std=0.1) if case["affine"] else None
        s["y"] = torch.empty_like(s["x"])
        if kind == "norm_train":
            s["dy"] = r.normal(rows, channels).to(dt)
            s["grads"] = [torch.empty_like(s["x"]), torch.empty_like(s["x"]) if case["gate"] else None,
                          zeros(channels) if case["affine"] else None, zeros(channels) if case["affine"] else None]
        return s
    B, T, H, H_kv, d_k, d_v = (case[x] for x in ("B", "T", "H", "H_kv", "d_k", "d_v"))
    lead = (B,) if kind == "step" else (B, T)
    s["q"] = r.normal(*lead, H, d_k).to(dt)
    s["k"] = _unit(r.normal(*lead, H_kv, d_k)).to(dt)
    s["v"] = r.normal(*lead, H_kv, d_v).to(dt)
    s["log_decay"] = -torch.exp(r.uniform(math.log(1.0 / 4096), math.log(0.5), H))
    s["scale"] = d_k ** -0.5
    s["o"] = zeros(*lead, H, d_v, dtype=dt)
    if kind == "step":
        s["S"] = r.normal(B, H, d_k, d_v, std=0.02)
        return s
    s["lens"] = (r.uniform(0, 1, B) * (T + 1)).to(torch.int32).clamp_(max=T) if case["ragged"] else None
    s["S0"] = r.normal(B, H, d_k, d_v, std=0.02) if case["state"] else None
    s["S_T"] = zeros(B, H, d_k, d_v)
    if kind == "train":
        s["d_o"] = r.normal(B, T, H, d_v).to(dt)
        s["dS_T"] = r.normal(B, H, d_k, d_v, std=0.1) if case["state"] else None
        s["grads"] = [torch.zeros_like(s[x]) for x in ("q", "k", "v")] + [zeros(B, H, d_k, d_v)]
    return s


# ------------------------------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits, powers of the decays and angles in 64
# ------------------------------------------------------------------------------------------------
def _power(log_decay, n):
    """exp(n log_decay) for n >= 0, zero for n < 0; heads in front."""
    x = torch.exp(log_decay.double().view(-1, *([1] * n.dim())) * n.clamp(min=0).double())
    return torch.where(n >= 0, x, torch.zeros_like(x)).float()


def _heads(x, H, T_pad=None):
    """[B, T, heads, d] -> fp32 [B, H, T, d], shared heads repeated, padded with zeros to T_pad tokens."""
    x = x.float().permute(0, 2, 1, 3)
    if x.shape[1] != H:
        x = x.repeat_interleave(H // x.shape[1], dim=1)
    if T_pad is not None and T_pad != x.shape[2]:
        x = torch.cat([x, x.new_zeros(x.shape[0], H, T_pad - x.shape[2], x.shape[3])], dim=2)
    return x


def _within(x, lens):
    """Rows behind a sequence's end set to zero ([B, H, T, d])."""
    if lens is None:
        return x
    return torch.where((torch.arange(x.shape[2], device=x.device) < lens.view(-1, 1)).view(x.shape[0], 1, -1, 1), x, torch.zeros_like(x))


def _scan(a, b, c, log_decay, reverse=False):
    """sum over i <= t of gamma^(t - i) (a_t . b_i) c_i, or over i >= t of gamma^(i - t): chunks against themselves, and
    against the earlier (later) chunks through their states b^T c."""
    B, H, T, da = a.shape
    n, dc, dev = T // C, c.shape[3], a.device
    a, b, c = (x.reshape(B, H, n, C, -1) for x in (a, b, c))
    i = torch.arange(C, device=dev)
    gap = i.view(-1, 1) - i.view(1, -1)
    inner = _power(log_decay, -gap if reverse else gap)                                    # [H, C, C]
    out = ((a @ b.transpose(-1, -2)) * inner.view(1, H, 1, C, C)) @ c
    if n > 1:
        w = _power(log_decay, i if reverse else C - 1 - i)                                 # to the chunk's edge
        state = (b * w.view(1, H, 1, C, 1)).transpose(-1, -2) @ c                          # [B, H, n, da, dc]
        j = torch.arange(n, device=dev)
        apart = (j.view(1, -1) - j.view(-1, 1) if reverse else j.view(-1, 1) - j.view(1, -1)) - 1
        far = torch.where(apart >= 0, apart * C, apart)
        state = (_power(log_decay, far).view(1, H, n, n) @ state.reshape(B, H, n, da * dc)).reshape(B, H, n, da, dc)
        e = _power(log_decay, C - i if reverse else i + 1)
        out = out + (a * e.view(1, H, 1, C, 1)) @ state
    return out.reshape(B, H, T, dc)


def _tokens(x, T, dt):
    return x[:, :, :T].permute(0, 2, 1, 3).to(dt).contiguous()


def _shared(x, H_kv):
    """Gradients of shared heads: the sum over the query heads that read them ([B, H, T, d] -> [B, H_kv, T, d])."""
    B, H, T, d = x.shape
    return x if H == H_kv else x.view(B, H_kv, H // H_kv, T, d).sum(2)


def _plain_step(s):
    H, dt = s["q"].shape[1], s["q"].dtype
    rep = lambda x: x.float().repeat_interleave(H // x.shape[1], dim=1)  # noqa: E731
    gamma = torch.exp(s["log_decay"].double()).float().view(1, -1, 1, 1)
    S = s["S"]
    S.mul_(gamma).add_(rep(s["k"]).unsqueeze(-1) * rep(s["v"]).unsqueeze(-2))
    o = (S * s["q"].float().unsqueeze(-1)).sum(-2) * s["scale"]
    return o.to(dt), S


def _plain_linear(s):
    case, ld, lens, scale = s["case"], s["log_decay"], s["lens"], s["scale"]
    B, T, H, H_kv, dt = case["B"], case["T"], case["H"], case["H_kv"], s["q"].dtype
    T_pad = -(-T // C) * C
    length = torch.full((B,), T, device="cuda", dtype=torch.int32) if lens is None else lens
    t = torch.arange(T_pad, device="cuda")
    q, k, v = (_within(_heads(s[x], H, T_pad), lens) for x in ("q", "k", "v"))
    since = _power(ld, t + 1).view(1, H, T_pad, 1)                                         # gamma^(t + 1): what is left of S0
    left = (length.view(-1, 1) - 1 - t).clamp(min=-1)                                      # tokens still to come
    until = _power(ld, left).permute(1, 0, 2).unsqueeze(-1)                                # [B, H, T, 1]
    whole = _power(ld, length).t().reshape(B, H, 1, 1)
    o = _scan(q, k, v, ld)
    S_T = (k * until).transpose(-1, -2) @ v
    if s["S0"] is not None:
        o = o + (q * since) @ s["S0"]
        S_T = S_T + whole * s["S0"]
    out = [_tokens(_within(o * scale, lens), T, dt), S_T]
    if case["kind"] == "prefill":
        return tuple(out)
    g = _within(_heads(s["d_o"], H, T_pad), lens)
    dq = _scan(g, v, k, ld) * scale
    dk = _scan(v, g, q, ld, reverse=True) * scale
    dv = _scan(k, q, g, ld, reverse=True) * scale
    dS0 = (q * since).transpose(-1, -2) @ g * scale
    if s["S0"] is not None:
        dq = dq + (g * since) @ s["S0"].transpose(-1, -2) * scale
    if s["dS_T"] is not None:
        dk = dk + (v * until) @ s["dS_T"].transpose(-1, -2)
        dv = dv + (k * until) @ s["dS_T"]
        dS0 = dS0 + whole * s["dS_T"]
    out += [_tokens(_within(dq, lens), T, dt), _tokens(_within(_shared(dk, H_kv), lens), T, dt),
            _tokens(_within(_shared(dv, H_kv), lens), T, dt), dS0]
    return tuple(out)


def _plain_rotary(s):
    case = s["case"]
    rot, sign = case["rot"], -1.0 if case["inverse"] else 1.0
    counts = s["positions"].long().unsqueeze(-1) * s["turns"]                               # modulo 2^64: one turn
    angle = counts.double() * (TURN / 2.0 ** 64)
    cos = (torch.cos(angle) * s["amplitude"]).float().unsqueeze(2)
    sin = (torch.sin(angle) * (s["amplitude"] * sign)).float().unsqueeze(2)

    def turned(x):
        y = x.float()
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["layout"] == "pairs" else (y[..., :rot // 2], y[..., rot // 2:rot])
        re, im = a * cos - b * sin, a * sin + b * cos
        head = torch.stack([re, im], dim=-1).flatten(-2) if case["layout"] == "pairs" else torch.cat([re, im], dim=-1)
        return torch.cat([head, y[..., rot:]], dim=-1).to(x.dtype)

    return turned(s["q"]), turned(s["k"])


def _plain_norm(s):
    case, x = s["case"], s["x"]
    rows, G, D, dt = case["rows"], case["groups"], case["width"], s["x"].dtype
    silu = case["act"] == "silu"
    x = x.float().view(rows, G, D)
    x = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = (x * rstd).view(rows, G * D)
    z = n if s["weight"] is None else n * s["weight"] + s["bias"]
    h = s["gate"].float() if case["gate"] else z                    # what the activation acts on
    sig = 1.0 / (1.0 + torch.exp(-h)) if silu else None
    a = h * sig if silu else h
    y = z * a if case["gate"] else a
    if case["kind"] == "norm":
        return (y.to(dt),)
    dy = s["dy"].float()
    slope = sig * (1.0 + h * (1.0 - sig)) if silu else torch.ones_like(h)
    dgate = (dy * z * slope).to(dt) if case["gate"] else None
    dz = dy * a if case["gate"] else dy * slope
    dn = (dz if s["weight"] is None else dz * s["weight"]).view(rows, G, D)
    nv = n.view(rows, G, D)
    dx = rstd * (dn - dn.mean(-1, keepdim=True) - nv * (dn * nv).mean(-1, keepdim=True))
    dw = (dz * n).sum(0) if s["weight"] is not None else None
    db = dz.sum(0) if s["weight"] is not None else None
    return y.to(dt), dx.view(rows, G * D).to(dt), dgate, dw, db


# ------------------------------------------------------------------------------------------------
# a pass
# ------------------------------------------------------------------------------------------------
def _workspace(s, name, size):
    """Scratch that a program allocates once for its sizes and keeps."""
    if name not in s:
        s[name] = torch.empty(size, device="cuda", dtype=torch.uint8) if size else None
    return s[name]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2607_11897_b200 as sfda
        if kind == "step":
            sfda.sfda_linear_step(s["q"], s["k"], s["v"], s["log_decay"], s["S"], s["o"], s["scale"])
            return s["o"], s["S"]
        if kind == "rotary":
            sfda.sfda_rotary(s["q"], s["k"], s["positions"], s["turns"], s["q_out"], s["k_out"],
                             sfda.SFDA_ROTARY_PAIRS if case["layout"] == "pairs" else sfda.SFDA_ROTARY_HALVES, s["amplitude"],
                             case["inverse"])
            return s["q_out"], s["k_out"]
        if kind in ("norm", "norm_train"):
            act = sfda.SFDA_ACT_SILU if case["act"] == "silu" else sfda.SFDA_ACT_NONE
            sfda.sfda_group_norm(s["x"], s["weight"], s["bias"], s["gate"], s["y"], case["groups"], EPS, act)
            if kind == "norm":
                return (s["y"],)
            dx, dgate, dw, db = s["grads"]
            ws = _workspace(s, "ws", sfda.sfda_group_norm_backward_workspace_bytes(case["rows"], case["groups"] * case["width"]))
            sfda.sfda_group_norm_backward(s["x"], s["weight"], s["bias"], s["gate"], s["dy"], dx, dw, db, dgate, case["groups"], EPS,
                                          act, ws)
            return s["y"], dx, dgate, dw, db
        code = sfda.SFDA_BF16 if case["dtype"] == "bf16" else sfda.SFDA_F32
        sizes = tuple(case[x] for x in ("B", "T", "H", "H_kv", "d_k", "d_v")) + (code,)
        ws = _workspace(s, "ws", sfda.sfda_linear_workspace_bytes(*sizes))
        sfda.sfda_linear_forward(s["q"], s["k"], s["v"], s["log_decay"], s["lens"], s["S0"], s["o"], s["S_T"], s["scale"], ws)
        if kind == "prefill":
            return s["o"], s["S_T"]
        bws = _workspace(s, "bws", sfda.sfda_linear_backward_workspace_bytes(*sizes))
        dq, dk, dv, dS0 = s["grads"]
        sfda.sfda_linear_backward(s["q"], s["k"], s["v"], s["log_decay"], s["lens"], s["S0"], s["d_o"], s["dS_T"], dq, dk, dv, dS0,
                                  s["scale"], bws)
        return s["o"], s["S_T"], dq, dk, dv, dS0
    if kind == "step":
        return _plain_step(s)
    if kind == "rotary":
        return _plain_rotary(s)
    if kind in ("norm", "norm_train"):
        return _plain_norm(s)
    return _plain_linear(s)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    e, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "rotary":
        n = case["B"] * case["T"] * (case["H"] + case["H_kv"])
        return {"bytes": 2 * n * case["d"] * e + 4 * case["B"] * case["T"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    if kind in ("norm", "norm_train"):
        n, ch = case["rows"] * case["groups"] * case["width"], case["groups"] * case["width"]
        moved, params = 3 if case["gate"] else 2, 8 * ch if case["affine"] else 0
        if kind == "norm":
            return {"bytes": n * moved * e + params, "flops": 12 * n}
        # x, the gate and dy are read once; y, dx and the gate's gradient are written
        return {"bytes": n * (moved + (3 if case["gate"] else 2)) * e + 2 * params, "flops": 40 * n}
    B, T, H, H_kv, d_k, d_v = (case[x] for x in ("B", "T", "H", "H_kv", "d_k", "d_v"))
    state = 4 * B * H * d_k * d_v
    inputs, o = B * T * (H * d_k + H_kv * (d_k + d_v)) * e, B * T * H * d_v * e
    once = 4 * B * T * H * d_k * d_v                  # one product of a token with the state and one update of it
    if kind == "step":
        return {"bytes": inputs + o + 2 * state, "flops": once}
    share = 0.5 if case["ragged"] else 1.0            # of the rows, on average, lie within their sequence
    forward = share * (inputs + o) + state * (2 if case["state"] else 1)
    if kind == "prefill":
        return {"bytes": forward, "flops": share * once}
    # the gradients of a row: the state and its adjoint once more, and a product with either for each of dq, dk, dv
    return {"bytes": forward + share * (inputs + o) + state * (2 if case["state"] else 1), "flops": share * 3.5 * once}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits, token by token
# ------------------------------------------------------------------------------------------------
def _exact_linear(s):
    case, lens = s["case"], s["lens"] if "lens" in s else None
    H, scale, train = case["H"], s["scale"], case["kind"] == "train"
    full = lambda x: x.double().repeat_interleave(H // x.shape[2], dim=2)  # noqa: E731
    q, k, v = full(s["q"]), full(s["k"]), full(s["v"])
    B, T, _, d_k = q.shape
    d_v = v.shape[-1]
    gamma = torch.exp(s["log_decay"].double()).view(1, H, 1, 1).expand(B, H, 1, 1).reshape(B * H, 1, 1)
    S = torch.zeros(B * H, d_k, d_v, device="cuda", dtype=torch.float64) if s["S0"] is None else s["S0"].double().reshape(B * H, d_k, d_v)
    ends = None if lens is None else lens.view(B, 1).expand(B, H).reshape(B * H, 1, 1)
    keep = lambda t, new, old: new if ends is None else torch.where(t < ends, new, old)  # noqa: E731
    o = torch.zeros(B, T, H, d_v, device="cuda", dtype=torch.float64)
    dq = torch.zeros_like(q) if train else None
    g = s["d_o"].double() if train else None
    at = lambda x, t: x[:, t].reshape(B * H, x.shape[-1])  # noqa: E731
    for t in range(T):
        new = torch.baddbmm(gamma * S, at(k, t).unsqueeze(2), at(v, t).unsqueeze(1))
        out = torch.bmm(at(q, t).unsqueeze(1), new).squeeze(1) * scale
        o[:, t] = keep(t, out.unsqueeze(1), torch.zeros_like(out).unsqueeze(1)).view(B, H, d_v)
        if train:
            d = torch.bmm(new, at(g, t).unsqueeze(2)).squeeze(2) * scale
            dq[:, t] = keep(t, d.unsqueeze(1), torch.zeros_like(d).unsqueeze(1)).view(B, H, d_k)
        S = keep(t, new, S)
    if not train:
        return o, S.view(B, H, d_k, d_v)
    G = torch.zeros_like(S) if s["dS_T"] is None else s["dS_T"].double().reshape(B * H, d_k, d_v)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    for t in range(T - 1, -1, -1):
        new = torch.baddbmm(G, at(q, t).unsqueeze(2), at(g, t).unsqueeze(1), alpha=scale)
        a, b = torch.bmm(new, at(v, t).unsqueeze(2)).squeeze(2), torch.bmm(at(k, t).unsqueeze(1), new).squeeze(1)
        dk[:, t] = keep(t, a.unsqueeze(1), torch.zeros_like(a).unsqueeze(1)).view(B, H, d_k)
        dv[:, t] = keep(t, b.unsqueeze(1), torch.zeros_like(b).unsqueeze(1)).view(B, H, d_v)
        G = keep(t, gamma * new, G)
    H_kv = case["H_kv"]
    group = lambda x: x.view(B, T, H_kv, H // H_kv, x.shape[-1]).sum(3)  # noqa: E731
    return o, S.view(B, H, d_k, d_v), dq, group(dk), group(dv), G.view(B, H, d_k, d_v)


def _exact_step(s):
    H = s["q"].shape[1]
    full = lambda x: x.double().repeat_interleave(H // x.shape[1], dim=1)  # noqa: E731
    S = s["S"].double() * torch.exp(s["log_decay"].double()).view(1, H, 1, 1)
    S = S + torch.einsum("bhk,bhv->bhkv", full(s["k"]), full(s["v"]))
    return torch.einsum("bhk,bhkv->bhv", s["q"].double(), S) * s["scale"], S


def _exact_rotary(s):
    case = s["case"]
    angle = s["positions"].double().unsqueeze(-1) * torch.from_numpy(_frequencies(case)).cuda()
    turn = torch.polar(torch.full_like(angle, s["amplitude"]), -angle if case["inverse"] else angle).unsqueeze(2)
    out = []
    for x in (s["q"], s["k"]):
        y, half = x.double().clone(), case["rot"] // 2
        re, im = (slice(0, case["rot"], 2), slice(1, case["rot"], 2)) if case["layout"] == "pairs" else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(y[..., re], y[..., im]) * turn
        y[..., re], y[..., im] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_norm(s):
    """The forward from its definition; the gradients by automatic differentiation of it in 64 bits."""
    case, train = s["case"], s["case"]["kind"] == "norm_train"
    leaf = lambda x: None if x is None else x.double().requires_grad_(train)  # noqa: E731
    x, gate, w, b = leaf(s["x"]), leaf(s["gate"]), leaf(s["weight"]), leaf(s["bias"])
    g = x.view(case["rows"], case["groups"], case["width"])
    var, mean = torch.var_mean(g, dim=-1, correction=0, keepdim=True)
    z = ((g - mean) / (var + EPS).sqrt()).reshape(x.shape)
    z = z if w is None else z * w + b
    act = (lambda h: h * torch.sigmoid(h)) if case["act"] == "silu" else (lambda h: h)
    y = act(z) if gate is None else z * act(gate)
    if not train:
        return (y,)
    got = torch.autograd.grad(y, [p for p in (x, gate, w, b) if p is not None], s["dy"].double())
    got = dict(zip([n for n, p in (("x", x), ("gate", gate), ("w", w), ("b", b)) if p is not None], got))
    return y.detach(), got["x"], got.get("gate"), got.get("w"), got.get("b")


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "step":
        return _exact_step(s)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    if case["kind"] in ("norm", "norm_train"):
        return _exact_norm(s)
    return _exact_linear(s)
