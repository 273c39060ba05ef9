"""The operators of a language model's layer that this library offers beside
its integer GEMMs and its attention core, over the sizes and data types that
programs give them: the calls themselves (`own`) and the same operators in
elementary torch operations.

A case is a dict of plain values; `op` names the operator:

  linear    a layer's projection with 8-bit weights: activations are quantised
            to 8 bits with one scale a token, multiplied with [N][K] weights
            with one scale an output channel, and come back in their own type
  product   the 8-bit product alone, on operands quantised beforehand
  attn      linear attention with a decay a head over a prompt: state in
            (`state`), state out, sequences of their own length (`ragged`)
  step      the same for one token a sequence; updates the state
  grad      the gradients of `attn`
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # one user's next token through a square projection: bound by reading the weights once
        dict(name="linear_1x4096", op="linear", dt="bf16", M=1, N=4096, K=4096, bias=False),
        # the next tokens of two dozen users through a wide projection
        dict(name="linear_24x8192", op="linear", dt="bf16", M=24, N=8192, K=4096, bias=True),
        # sizes that fit no tile, rows that start at odd addresses
        dict(name="linear_ragged", op="linear", dt="f16", M=777, N=1000, K=1501, bias=True),
        # a prompt of 2048 tokens through a wide projection
        dict(name="linear_2048", op="linear", dt="bf16", M=2048, N=8192, K=4096, bias=True),
        # the largest product, on activations quantised beforehand
        dict(name="product_8192", op="product", dt="bf16", M=8192, N=8192, K=8192, bias=False),
        # a short prompt of a small model, half precision
        dict(name="attn_512_d64", op="attn", dt="f16", B=1, H=16, L=512, dk=64, dv=64, state=False, ragged=False),
        # long prompts continued from a state, 32 heads of 128
        dict(name="attn_8192_d128", op="attn", dt="bf16", B=2, H=32, L=8192, dk=128, dv=128, state=True,
             ragged=False),
        # a padded batch of unlike lengths, odd head sizes, single precision
        dict(name="attn_ragged_f32", op="attn", dt="f32", B=8, H=8, L=1999, dk=96, dv=80, state=True, ragged=True),
        # one user's next token: 16 small states, bound by its launch
        dict(name="step_1_d64", op="step", dt="bf16", B=1, H=16, dk=64, dv=64),
        # the next tokens of 64 users: bound by reading and writing the states
        dict(name="step_64_d128", op="step", dt="bf16", B=64, H=32, dk=128, dv=128),
        # a training step's sequences
        dict(name="grad_4096_d128", op="grad", dt="bf16", B=4, H=16, L=4096, dk=128, dv=128, state=False,
             ragged=False),
        # a small padded training batch in single precision, with the gradient of its initial state
        dict(name="grad_ragged_f32", op="grad", dt="f32", B=3, H=6, L=1023, dk=64, dv=64, state=True, ragged=True),
    ]


def _log(rng, lo, hi):
    """An integer from [lo, hi], even over its logarithm; about half of them odd or ragged."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 32 and rng.random() < 0.5:
        v = v // 16 * 16
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "product", "attn", "attn", "attn", "step", "step", "grad", "grad"])
    dt = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("linear", "product"):
        while True:
            M = rng.choice([_log(rng, 1, 64), _log(rng, 64, 8192)])
            N, K = _log(rng, 32, 8192), _log(rng, 32, 8192)
            if rng.random() < 0.75:          # most models' widths are whole vectors
                K = (K + 31) // 32 * 32
            if M * N * K <= 2 ** 38:
                break
        return dict(op=op, dt=dt, M=M, N=N, K=K, bias=rng.random() < 0.5)
    d = [32, 48, 64, 64, 80, 96, 128, 128, 128]
    dk = rng.choice(d + [256])
    dv = rng.choice([dk, dk, rng.choice(d + [256])])
    if op == "step":
        while True:
            B, H = _log(rng, 1, 256), _log(rng, 1, 64)
            if B * H * dk * dv <= 2 ** 25:
                break
        return dict(op=op, dt=dt, B=B, H=H, dk=dk, dv=dv)
    while True:
        B, H, L = _log(rng, 1, 32), _log(rng, 1, 64), _log(rng, 1, 16384)
        if 2 ** 10 <= B * H * L * (dk + dv) <= (2 ** 26 if op == "attn" else 2 ** 25) and dt != "f32" or \
                2 ** 10 <= B * H * L * (dk + dv) <= 2 ** 24:
            break
    return dict(op=op, dt=dt, B=B, H=H, L=L, dk=dk, dv=dv, state=rng.random() < 0.5, ragged=B > 1 and rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _quantized(x):
    """[rows][cols] float32 as 8-bit values and one scale a row (the weights as a program holds them)."""
    s = x.abs().amax(1) / 127
    return torch.round(x / s[:, None]).clamp(-127, 127).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T = TYPES[case["dt"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = dict(case)
    if case["op"] in ("linear", "product"):
        M, N, K = case["M"], case["N"], case["K"]
        # a few channels carry most of the size, as activations of such layers do
        x = normal(M, K) * (1 + 4 * (torch.rand(K, generator=g, device="cuda") > 0.98))
        s["w"], s["scale_w"] = _quantized(normal(N, K) * K ** -0.5)
        s["bias_t"] = normal(N) * 0.1 if case["bias"] else None
        if case["op"] == "product":
            s["a"], s["scale_a"] = _quantized(x)
        else:
            s["x"] = x.to(T)
        return s
    B, H, dk, dv = (case[n] for n in ("B", "H", "dk", "dv"))
    rows = (case["L"],) if "L" in case else ()
    s["q"], s["k"], s["v"] = normal(B, H, *rows, dk).to(T), normal(B, H, *rows, dk).to(T), normal(B, H, *rows, dv).to(T)
    # decays from one half to a memory of some 200 tokens, another one for each head
    h = torch.arange(H, device="cuda", dtype=torch.float32) / max(H - 1, 1)
    s["log_decay"] = -torch.exp2(-1 - 7 * h) * (0.9 + 0.2 * torch.rand(H, generator=g, device="cuda"))
    s["scale"] = dk ** -0.5
    if case["op"] == "step":
        s["state_t"] = normal(B, H, dk, dv)
        return s
    s["state_t"] = normal(B, H, dk, dv) if case["state"] else None
    if case["op"] == "grad":
        s["do"] = normal(B, H, *rows, dv).to(T)
        s["d_state"] = normal(B, H, dk, dv) * 0.1 if case["state"] else None
    s["lens"] = None
    if case["ragged"]:
        n = torch.randint(0, case["L"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        n[0] = case["L"]
        s["lens"] = n
    # rows behind a sequence's end stay as they are: the buffers hold zeros there
    zeros = lambda t: torch.zeros_like(t)  # noqa: E731
    s["out"] = zeros(s["v"]) if case["op"] == "attn" else [zeros(s["q"]), zeros(s["k"]), zeros(s["v"])]
    return s


# ---------------------------------------------------------------------------
# the operators in elementary operations
# ---------------------------------------------------------------------------
def _plain_product(a, sa, w, sw, bias, T):
    y = (a.float() @ w.float().t()) * sa[:, None] * sw[None, :]
    if bias is not None:
        y = y + bias
    return y.to(T)


def _powers(g, n):
    """exp(g n) [H][...] for exponents n >= 0 (any shape), 0 where n < 0."""
    n = n.double()
    e = torch.exp(g.double().view(-1, *([1] * n.dim())) * n.clamp_min(0))
    return torch.where(n < 0, torch.zeros_like(e), e).float()


def _core(x, y, z, g):
    """sum over j <= i of exp(g (i - j)) (x_i . y_j) z_j, in chunks of 64 tokens."""
    C = 64
    B, H, L, dx = x.shape
    n = -(-L // C)
    cut = lambda t: torch.nn.functional.pad(t, (0, 0, 0, n * C - L)).reshape(B, H, n, C, -1)  # noqa: E731
    x, y, z = cut(x), cut(y), cut(z)
    i = torch.arange(C, device=x.device)
    near = (x @ y.transpose(-1, -2)) * _powers(g, i[:, None] - i[None, :])[:, None] @ z
    per = y.transpose(-1, -2) @ (z * _powers(g, C - 1 - i)[:, None, :, None])        # a chunk's own state
    c = torch.arange(n, device=x.device)
    before = (_powers(g, C * (c[:, None] - 1 - c[None, :])) @ per.reshape(B, H, n, -1)).reshape(per.shape)
    far = (x * _powers(g, i + 1)[:, None, :, None]) @ before
    return (near + far).reshape(B, H, n * C, -1)[:, :, :L]


def _plain_attn(x, y, z, g, scale, state, lens, back):
    """The recurrence over the sequences' own lengths, from their ends to their starts where `back`:
    outputs and the state after the last token taken (float32)."""
    B, H, L, dx = x.shape
    x, y, z = x.float(), y.float(), z.float()
    i = torch.arange(L, device=x.device)
    n = torch.full((B,), L, device=x.device) if lens is None else lens.long()
    seen = (i[None, :] < n[:, None])[:, None, :, None]
    # the values are put aside, not multiplied by zero: what stands behind the end may be anything
    x, y, z = (torch.where(seen, t, torch.zeros_like(t)) for t in (x, y, z))
    if back:
        o = _core(x.flip(2), y.flip(2), z.flip(2), g).flip(2)
        first = n[:, None] - 1 - i[None, :]
        last = i[None, :] + 1 + 0 * n[:, None]
    else:
        o = _core(x, y, z, g)
        first = i[None, :] + 1 + 0 * n[:, None]
        last = n[:, None] - 1 - i[None, :]
    end = y.transpose(-1, -2) @ (z * _powers(g, last).transpose(0, 1)[..., None]) * scale
    o = o * scale
    if state is not None:
        w = _powers(g, first).transpose(0, 1)[..., None]
        o = o + (x * w) @ state * (1 if back else scale)
        end = (end if back else end / scale) + _powers(g, n).transpose(0, 1)[..., None, None] * state
    elif not back:
        end = end / scale
    return torch.where(seen, o, torch.zeros_like(o)), end


def run(s):
    if own:
        from paper_2606_09905_amd import qx
    op, T = s["op"], TYPES[s["dt"]]
    if op == "linear":
        if own:
            return qx.linear_i8(s["x"], s["w"], s["scale_w"], bias=s["bias_t"])
        x = s["x"].float()
        # (a GPU tensor over a plain number is multiplied by its rounded reciprocal: a step off in
        # one scale of twenty, and with it values next to a half on the other side)
        sa = (x.abs().amax(1).double() / 127).float()
        a = torch.round(x / sa[:, None]).clamp(-127, 127)
        return _plain_product(a, sa, s["w"], s["scale_w"], s["bias_t"], T)
    if op == "product":
        if own:
            return qx.qgemm_i8_scaled(s["a"], s["w"], s["scale_a"], s["scale_w"], bias=s["bias_t"], dtype=T)
        return _plain_product(s["a"], s["scale_a"], s["w"], s["scale_w"], s["bias_t"], T)
    q, k, v, g, scale = s["q"], s["k"], s["v"], s["log_decay"], s["scale"]
    if op == "step":
        if own:
            return qx.lin_attn_step(q, k, v, g, s["state_t"], scale=scale), s["state_t"]
        S = s["state_t"]
        S.mul_(torch.exp(g)[None, :, None, None]).add_(k.float()[..., :, None] * v.float()[..., None, :])
        return ((q.float()[..., None, :] @ S)[..., 0, :] * scale).to(T), S
    if op == "attn":
        if own:
            return qx.lin_attn(q, k, v, g, scale=scale, state=s["state_t"], lens=s["lens"], out=s["out"])
        o, end = _plain_attn(q, k, v, g, scale, s["state_t"], s["lens"], False)
        return o.to(T), end
    do, S0, dS = s["do"], s["state_t"], s["d_state"]
    if own:
        got = qx.lin_attn_backward(q, k, v, do, g, scale=scale, state=S0, d_state=dS, lens=s["lens"], out=s["out"])
        return got if S0 is not None else got[:3]
    flip = lambda t: None if t is None else t.transpose(-1, -2)  # noqa: E731
    dq, _ = _plain_attn(do, v, k, g, scale, flip(S0), s["lens"], False)
    dk, _ = _plain_attn(v, do, q, g, scale, flip(dS), s["lens"], True)
    dv, dS0 = _plain_attn(k, q, do, g, scale, dS, s["lens"], True)
    return (dq.to(T), dk.to(T), dv.to(T)) + ((dS0,) if S0 is not None else ())


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    es = 4 if case["dt"] == "f32" else 2
    if case["op"] in ("linear", "product"):
        M, N, K = case["M"], case["N"], case["K"]
        a = M * K * (es if case["op"] == "linear" else 1) + (4 * M if case["op"] == "product" else 0)
        return {"bytes": a + N * K + 4 * N * (2 if case["bias"] else 1) + M * N * es, "flops": 2 * M * N * K}
    B, H, dk, dv = (case[n] for n in ("B", "H", "dk", "dv"))
    heads, S = B * H, 4 * B * H * dk * dv
    if case["op"] == "step":
        return {"bytes": 2 * S + heads * (2 * dk + 2 * dv) * es, "flops": 5 * heads * dk * dv}
    tokens = heads * case["L"] / (2 if case["ragged"] else 1)     # lengths are even over [0, L]
    states = S * (2 if case["state"] else 1)
    if case["op"] == "attn":
        return {"bytes": tokens * (2 * dk + 2 * dv) * es + states, "flops": 4 * tokens * dk * dv}
    return {"bytes": tokens * (4 * dk + 3 * dv) * es + (3 * S if case["state"] else 0), "flops": 10 * tokens * dk * dv}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("linear", "product"):
        if op == "linear":
            # the scale and the 8-bit values are defined by single-precision arithmetic, each
            # quotient rounded once: from 64 bits, which hold it far enough for that
            x = s["x"].to(torch.float64)
            sa = torch.div(torch.max(torch.abs(x), dim=1).values, 127.0).to(torch.float32)
            a = torch.div(x, sa.to(torch.float64).unsqueeze(1)).to(torch.float32)
            a = torch.clamp(torch.round(a), -127, 127)
        else:
            a, sa = s["a"], s["scale_a"]
        y = torch.mm(a.double(), s["w"].double().t().contiguous())      # whole numbers below 2^53
        y = y * torch.outer(sa.double(), s["scale_w"].double())
        return y if s["bias_t"] is None else y + s["bias_t"].double()[None, :]
    q, k, v, g = (s[n].double() for n in ("q", "k", "v", "log_decay"))
    scale, S0 = s["scale"], s["state_t"]
    if op == "step":
        S = S0.double() * torch.exp(g)[None, :, None, None] + torch.einsum("bha,bhc->bhac", k, v)
        return scale * torch.einsum("bha,bhac->bhc", q, S), S
    B, H, L, dk = q.shape
    dv = v.shape[-1]
    n = [L] * B if s["lens"] is None else [int(t) for t in s["lens"].cpu()]
    if B * H * L * L > 2 ** 36:
        return None
    if op == "attn":
        o = torch.zeros(B, H, L, dv, dtype=torch.float64, device="cuda")
        S = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda")
    else:
        do = s["do"].double()
        dq, dkk, dvv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dS0 = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda")
    for b in range(B):
        m = n[b]
        i = torch.arange(m, device="cuda", dtype=torch.float64)
        for h in range(H):
            D = torch.exp(g[h] * (i[:, None] - i[None, :]).clamp_min(0)).tril()     # decay from j to i
            start, end = torch.exp(g[h] * (i + 1))[:, None], torch.exp(g[h] * (m - 1 - i))[:, None]
            Q, K, V = q[b, h, :m], k[b, h, :m], v[b, h, :m]
            init = None if S0 is None else S0[b, h].double()
            if op == "attn":
                r = torch.mm(torch.mm(Q, K.t()) * D, V)
                f = torch.mm(K.t(), end * V)
                if init is not None:
                    r = r + start * torch.mm(Q, init)
                    f = f + torch.exp(g[h] * m) * init
                o[b, h, :m], S[b, h] = scale * r, f
                continue
            dO = scale * do[b, h, :m]
            A, P = torch.mm(dO, V.t()) * D, torch.mm(Q, K.t()) * D
            gq, gk, gv = torch.mm(A, K), torch.mm(A.t(), Q), torch.mm(P.t(), dO)
            if init is not None:
                last = s["d_state"][b, h].double()
                gq = gq + start * torch.mm(dO, init.t())
                gk = gk + end * torch.mm(V, last.t())
                gv = gv + end * torch.mm(K, last)
                dS0[b, h] = torch.mm(Q.t(), start * dO) + torch.exp(g[h] * m) * last
            dq[b, h, :m], dkk[b, h, :m], dvv[b, h, :m] = gq, gk, gv
    if op == "attn":
        return o, S
    return (dq, dkk, dvv) + ((dS0,) if S0 is not None else ())
