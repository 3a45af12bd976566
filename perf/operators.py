"""Operators of a training step that this library's networks need: what is measured, and what it has to compute.

A drafter or a policy network is tuned on noised action chunks.  Its convolutions and projections are followed by a
GroupNorm with an activation (and FiLM vectors of the conditioning), channels last; what the backward pass needs of the
forward pass is kept in eight bits.  The operators are

  norm     y = scale * act(GroupNorm(x)) + bias, statistics kept, input and output saved in eight bits on request
  grad     its gradients: of x, of the affine vectors and of the FiLM vectors, from x or from its 8-bit copy
  save     the 8-bit copy of a tensor, and the tensor that it stands for
  weight   the gradient of a projection's or a convolution's weights and bias, its input read from the 8-bit copy

The 8-bit copy: each row is cut into blocks of 32 channels; a block holds whole numbers q, |q| <= 127, and one byte b, and
stands for q * 2^(b - 127); b is the smallest for which no rounded value exceeds 127 (within 1 .. 248), 255 for a block
with a value that is not finite, which is read back as NaN.  Rounding is to the nearest, halves to even.
"""
import functools

import torch

own = False      # False: plain torch forms; True: the calls that a user of this library makes

NORM, GRAD, SAVE, WEIGHT = "norm", "grad", "save", "weight"
BF16, FP32 = "bf16", "fp32"
EPS = 1e-5


def _norm(name, op, N, L, C, groups, dtype, act="mish", film=False, saved=False):
    """N sequences of L positions and C channels; saved: `norm` writes both 8-bit copies, `grad` reads x from its copy."""
    c = dict(op=op, N=N, L=L, C=C, groups=groups, dtype=dtype, act=act, film=film, saved=saved)
    return dict(c, name=name) if name else c


def _save(name, rows, C, dtype):
    c = dict(op=SAVE, rows=rows, C=C, dtype=dtype)
    return dict(c, name=name) if name else c


def _weight(name, N, L, K, out, taps, dtype):
    """N sequences of L rows, K channels in, `out` channels out, `taps` taps along the sequence (1: a projection)."""
    c = dict(op=WEIGHT, N=N, L=L, K=K, out=out, taps=taps, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # first level of the conv UNet, one chunk: the smallest call there is
        _norm("norm_one_chunk", NORM, 1, 16, 256, 8, BF16, film=True),
        # second level of the conv UNet, a batch of 4096 noised chunks, everything kept for the backward pass
        _norm("norm_batch", NORM, 4096, 16, 512, 8, BF16, film=True, saved=True),
        # a few long sequences in fp32, odd length, groups of ten channels
        _norm("norm_long", NORM, 3, 4099, 320, 32, FP32, act="silu"),
        # the gradients at the same places
        _norm("grad_one_chunk", GRAD, 1, 16, 256, 8, BF16, film=True),
        _norm("grad_batch", GRAD, 4096, 16, 512, 8, BF16, film=True, saved=True),
        _norm("grad_long", GRAD, 5, 2777, 200, 8, FP32, act="gelu"),
        # a small tensor of odd width, and the hidden layer of the serving transformer's MLP over a full batch of candidates
        _save("save_odd", 37, 100, FP32),
        _save("save_mlp", 45056, 2048, BF16),
        # a drafter's MLP over 24 chunks of 16 tokens; a kernel-5 convolution of the UNet; the serving transformer's MLP
        _weight("weight_small", 24, 16, 128, 512, 1, BF16),
        _weight("weight_conv", 1024, 16, 512, 512, 5, BF16),
        _weight("weight_mlp", 2816, 16, 512, 2048, 1, BF16),
        # fp32, odd everywhere
        _weight("weight_odd", 7, 143, 77, 130, 3, FP32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    """Another call of the same kinds: sizes spread over the logarithm of their ranges, within the largest listed case."""
    op = rng.choice((NORM, GRAD, SAVE, WEIGHT))
    dtype = rng.choice((BF16, BF16, FP32))
    if op in (NORM, GRAD):
        groups = rng.choice((1, 4, 8, 8, 16, 32))
        C = groups * rng.choice((_log_int(rng, 1, max(1, 1024 // groups)), 32, 64))
        L = rng.choice((_log_int(rng, 1, 4096), 4, 8, 16))
        L = max(L, -(-16 * groups // C))             # (a group of a few values keeps no direction for a gradient of x)
        N = _log_int(rng, 1, max(1, min(4096, (1 << 24) // (L * C))))
        return _norm(None, op, N, L, C, groups, dtype, rng.choice(("mish", "mish", "silu", "gelu", "none")),
                     rng.random() < 0.5, rng.random() < 0.5)
    if op == SAVE:
        C = rng.choice((_log_int(rng, 1, 4096), 256, 512, 1024, 2048))
        return _save(None, _log_int(rng, 1, max(1, min(65536, (45056 * 1024) // C))), C, dtype)
    taps = rng.choice((1, 1, 3, 5))
    K, out = (rng.choice((_log_int(rng, 8, 1024), 128, 256, 512)) for _ in range(2))
    L = rng.choice((_log_int(rng, 1, 512), 4, 8, 16))
    most = min(32768, (45056 * 512 * 2048) // (K * out * taps * (4 if dtype == FP32 else 1)))
    return _weight(None, max(1, _log_int(rng, 16, max(17, most)) // L), L, K, out, taps, dtype)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == BF16 else torch.float32


def _blocks(C):
    return (C + 31) // 32


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, rows, C, dtype):
    """What a convolution gives: channels of their own offset and width."""
    return (_randn(g, rows, C) * torch.exp(0.5 * _randn(g, C)) + 0.5 * _randn(g, C)).to(dtype)


# ------------------------------------------------------------------------------- plain forms
def _pack(x):
    """(q, b) of x [rows, C]."""
    rows, C = x.shape
    nb = _blocks(C)
    v = torch.zeros(rows, nb * 32, dtype=torch.float32, device=x.device)
    v[:, :C] = x
    v = v.view(rows, nb, 32)
    top = v.abs().amax(2)
    bad = ~torch.isfinite(v).all(2)
    top = torch.where(bad, torch.ones_like(top), top)
    mant, exp = torch.frexp(top)                                       # top = mant 2^exp, mant in [0.5, 1): 2^6 <= mant 2^7 < 2^7
    b = (exp + 120 + (torch.round(mant * 128.0) > 127.0)).clamp(1, 248)
    b = torch.where(top == 0, torch.ones_like(b), b)
    v = torch.where(bad[..., None], torch.zeros_like(v), v)
    q = torch.round(torch.ldexp(v.double(), (127 - b)[..., None])).clamp(-127, 127).to(torch.int8)
    b = torch.where(bad, torch.full_like(b, 255), b).to(torch.uint8)
    return q.view(rows, nb * 32)[:, :C].contiguous(), b


def _unpack(q, b, dtype):
    """What (q, b) stand for."""
    step = torch.ldexp(torch.ones_like(b, dtype=torch.float32), b.int() - 127)
    step = torch.where(b == 255, torch.full_like(step, float("nan")), step)
    return (q.float() * step.repeat_interleave(32, 1)[:, :q.shape[1]]).to(dtype)


def _sigmoid(z):
    return 1.0 / (1.0 + torch.exp(-z))


def _act(name, z):
    """(act(z), act'(z))"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        s = _sigmoid(z)
        return z * s, s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        k, c = 0.7978845608028654, 0.044715
        t = torch.tanh(k * (z + c * z * z * z))
        return 0.5 * z * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3.0 * c * z * z)
    t = torch.tanh(torch.log1p(torch.exp(-z.abs())) + torch.relu(z))     # mish: z tanh(softplus(z))
    return z * t, t + z * (1.0 - t * t) * _sigmoid(z)


def _plain_norm(s):
    c = s["case"]
    N, L, C, G = c["N"], c["L"], c["C"], c["groups"]
    v = s["x"].float().view(N, L, G, C // G)
    mean = v.mean((1, 3))
    d = v - mean[:, None, :, None]
    rstd = torch.rsqrt((d * d).mean((1, 3)) + EPS)
    a, _ = _act(c["act"], (d * rstd[:, None, :, None]).view(N, L, C) * s["gamma"] + s["beta"])
    if c["film"]:
        a = s["film"][:, None, :C] * a + s["film"][:, None, C:]
    out = dict(y=a.to(_dtype(c)), mean=mean, rstd=rstd)
    if c["saved"]:
        for k, t in (("saved_x", s["x"]), ("saved_y", out["y"])):
            out[k] = _unpack(*_pack(t.reshape(N * L, C)), _dtype(c))
    return out


def _plain_grad(s):
    c = s["case"]
    N, L, C, G = c["N"], c["L"], c["C"], c["groups"]
    x = _unpack(*s["saved_x"], torch.float32).view(N, L, C) if c["saved"] else s["x"].float()
    spread = lambda t: t.repeat_interleave(C // G, 1)[:, None, :]  # noqa: E731
    h = (x - spread(s["mean"])) * spread(s["rstd"])
    a, da = _act(c["act"], h * s["gamma"] + s["beta"])
    dy, out = s["dy"].float(), {}
    dz = dy * da
    if c["film"]:
        out["dfilm"] = torch.cat([(dy * a).sum(1), dy.sum(1)], 1)
        dz = dz * s["film"][:, None, :C]
    p, r = dz.sum(1), (dz * h).sum(1)                                     # [N, C]
    of_group = lambda t: spread((t * s["gamma"]).view(N, G, C // G).sum(2) / (L * (C // G)))  # noqa: E731
    dx = spread(s["rstd"]) * (dz * s["gamma"] - of_group(p) - h * of_group(r))
    return dict(out, dx=dx.to(_dtype(c)), dgamma=r.sum(0), dbeta=p.sum(0))


def _plain_weight(s):
    c = s["case"]
    N, L, K, out, taps = (c[k] for k in ("N", "L", "K", "out", "taps"))
    x = _unpack(*s["saved_x"], torch.float32).view(N, L, K)
    dy = s["dy"].float()
    side = torch.zeros(N, taps // 2, K, device=x.device)
    x = torch.cat([side, x, side], 1).unfold(1, L, 1).permute(1, 2, 0, 3).reshape(taps * K, N * L)     # [tap, in] x rows
    return dict(dW=(x @ dy).view(taps, K, out), db=dy.sum(0))


# ------------------------------------------------------------------------------- the cases
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, op, s = _dtype(case), case["op"], dict(case=case)
    empty = functools.partial(torch.empty, device="cuda")
    u8 = dict(dtype=torch.uint8)
    if op == SAVE:
        rows, C = case["rows"], case["C"]
        return dict(s, x=_activations(g, rows, C, t), back=empty(rows, C, dtype=t),
                    saved=(empty(rows, C, dtype=torch.int8), empty(rows, _blocks(C), **u8)))
    N, L = case["N"], case["L"]
    if op == WEIGHT:
        K, out, taps = case["K"], case["out"], case["taps"]
        x = _act("mish", _activations(g, N * L, K, torch.float32))[0].to(torch.bfloat16)      # what stands before a layer
        return dict(s, saved_x=_pack(x), dy=(_randn(g, N * L, out) * torch.exp(0.5 * _randn(g, out)) / N).to(t),
                    dW=empty(taps, K, out), db=empty(out), workspace=empty(WORKSPACE, **u8))
    C, G = case["C"], case["groups"]
    s["gamma"], s["beta"] = 1.0 + 0.1 * _randn(g, C), 0.1 * _randn(g, C)
    if case["film"]:
        s["film"] = 0.3 * _randn(g, N, 2 * C)
        s["film"][:, :C] += 1.0
    x = _activations(g, N * L, C, t)
    if op == NORM:
        s.update(x=x.view(N, L, C), y=empty(N, L, C, dtype=t), mean=empty(N, G), rstd=empty(N, G))
        for k in ("saved_x", "saved_y") if case["saved"] else ():
            s[k] = (empty(N * L, C, dtype=torch.int8), empty(N * L, _blocks(C), **u8))
            s["back_" + k] = empty(N * L, C, dtype=t)
        return s
    v = x.float().view(N, L, G, C // G)
    s["mean"] = v.mean((1, 3))
    s["rstd"] = torch.rsqrt(((v - s["mean"][:, None, :, None]) ** 2).mean((1, 3)) + EPS)
    if case["saved"]:
        s["saved_x"] = _pack(x)
    else:
        s["x"] = x.view(N, L, C)
    s.update(dy=_randn(g, N, L, C).to(t), dx=empty(N, L, C, dtype=t), dgamma=empty(C), dbeta=empty(C),
             workspace=empty(WORKSPACE, **u8))
    if case["film"]:
        s["dfilm"] = empty(N, 2 * C)
    return s


WORKSPACE = 64 << 20      # partial sums of the gradients: one buffer for all layers


def run(state):
    s, c = state, state["case"]
    if own:
        return _own_run(s, c)
    if c["op"] == NORM:
        return _plain_norm(s)
    if c["op"] == GRAD:
        return _plain_grad(s)
    if c["op"] == SAVE:
        return dict(back=_unpack(*_pack(s["x"]), _dtype(c)))
    return _plain_weight(s)


def _own_run(s, c):
    from paper_2512_15773_b200 import binding
    if c["op"] == SAVE:
        binding.checkpoint_pack(s["x"], s["saved"])
        binding.checkpoint_unpack(s["saved"], s["back"])
        return dict(back=s["back"])
    if c["op"] == WEIGHT:
        binding.weight_grad(s["saved_x"], s["dy"], s["dW"], s["workspace"], db=s["db"], length=c["L"])
        return dict(dW=s["dW"], db=s["db"])
    if c["op"] == NORM:
        binding.group_norm(s["x"], s["gamma"], s["beta"], c["groups"], s["y"], act=c["act"], film=s.get("film"), eps=EPS,
                           mean=s["mean"], rstd=s["rstd"], saved_x=s.get("saved_x"), saved_y=s.get("saved_y"))
        out = dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        for k in ("saved_x", "saved_y") if c["saved"] else ():
            binding.checkpoint_unpack(s[k], s["back_" + k])
            out[k] = s["back_" + k]
        return out
    binding.group_norm_grad(s["dy"], s.get("x"), s["gamma"], s["beta"], c["groups"], s["mean"], s["rstd"], s["dx"], s["dgamma"],
                            s["dbeta"], s["workspace"], act=c["act"], film=s.get("film"), dfilm=s.get("dfilm"),
                            saved_x=s.get("saved_x"))
    out = dict(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    return dict(out, dfilm=s["dfilm"]) if c["film"] else out


def work(case):
    """Inputs read once, outputs written once; an 8-bit copy takes 33 bytes for 32 values."""
    size = 2 if case["dtype"] == BF16 else 4
    if case["op"] == SAVE:
        n, m = case["rows"] * case["C"], case["rows"] * (case["C"] + _blocks(case["C"]))
        return dict(bytes=2 * size * n + 2 * m, flops=4 * n)            # written and read back
    if case["op"] == WEIGHT:
        M, K, out, taps = case["N"] * case["L"], case["K"], case["out"], case["taps"]
        return dict(bytes=M * (K + _blocks(K)) + size * M * out + 4 * (taps * K + 1) * out, flops=2 * taps * M * K * out)
    rows, C = case["N"] * case["L"], case["C"]
    n, copy = rows * C, rows * (C + _blocks(C))
    small = 8 * C + 8 * case["N"] * case["groups"] + (8 * case["N"] * C if case["film"] else 0)
    if case["op"] == NORM:
        more = 4 * copy + 2 * size * n if case["saved"] else 0              # both copies written, and read back
        return dict(bytes=2 * size * n + small + more, flops=20 * n)
    small += 8 * C + (8 * case["N"] * C if case["film"] else 0)
    return dict(bytes=2 * size * n + (copy if case["saved"] else size * n) + small, flops=40 * n)


# ------------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_copy(x):
    """The values that the 8-bit copy of x [rows, C] stands for, block by block of columns."""
    parts = []
    for c0 in range(0, x.shape[1], 32):
        v = x[:, c0:c0 + 32].double()
        top = v.abs().max(1, keepdim=True).values
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
        e = torch.where(2.0 ** e > top, e - 1, torch.where(2.0 ** (e + 1) <= top, e + 1, e)) - 6      # 64 <= top 2^-e < 128
        e = torch.where(torch.round(top * 2.0 ** -e) > 127, e + 1, e).clamp(-126, 121)
        parts.append((torch.round(v * 2.0 ** -e) * 2.0 ** e))
    return torch.cat(parts, 1)


def _exact_values(copy):
    q, b = copy
    return torch.cat([q[:, 32 * j:32 * j + 32].double() * 2.0 ** (b[:, j:j + 1].double() - 127) for j in range(b.shape[1])], 1)


def _exact_act(name, z):
    """act and its derivative in 64 bits; the derivative of Mish and SiLU through the logistic function's own."""
    if name == "none":
        return z, torch.ones_like(z)
    lg = torch.sigmoid(z)
    if name == "silu":
        return z * lg, lg + z * lg * (1 - lg)
    if name == "gelu":
        u = 0.7978845608028654 * (z + 0.044715 * z ** 3)
        return z * torch.sigmoid(2 * u), torch.sigmoid(2 * u) + z * 2 * torch.sigmoid(2 * u) * torch.sigmoid(-2 * u) * 0.7978845608028654 * (1 + 0.134145 * z ** 2)
    e = torch.exp(-z.abs())                                       # tanh(log(1 + e^z)) = (1 - w) / (1 + w) with w = (1 + e^z)^-2
    w = torch.where(z > 0, (e / (1 + e)) ** 2, (1 / (1 + e)) ** 2)
    t = torch.where(z > 0, (1 - w) / (1 + w), (e * e + 2 * e) / (e * e + 2 * e + 2))
    return z * t, t + z * lg * 4 * w / (1 + w) ** 2


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == SAVE:
        return dict(back=_exact_copy(s["x"]))
    if case["op"] == WEIGHT:
        N, L, taps = case["N"], case["L"], case["taps"]
        x, dy = _exact_values(s["saved_x"]).view(N, L, -1), s["dy"].double().view(N, L, -1)
        dW = []
        for tap in range(taps):
            o = tap - taps // 2                                     # output row l takes input row l + o
            lo, hi = max(0, -o), max(max(0, -o), min(L, L - o))
            dW.append(x[:, lo + o:hi + o].reshape(-1, case["K"]).T @ dy[:, lo:hi].reshape(-1, case["out"]))
        return dict(dW=torch.stack(dW), db=dy.sum((0, 1)))
    N, L, C, G = case["N"], case["L"], case["C"], case["groups"]
    w = C // G
    out = {k: [] for k in (("y", "mean", "rstd") if case["op"] == NORM else ("dx", "dgamma", "dbeta", "ds", "db"))}
    values = None if case["op"] == NORM else (_exact_values(s["saved_x"]).view(N, L, C) if case["saved"] else s["x"].double())
    for j in range(G):
        ch = slice(j * w, j * w + w)
        ga, be = s["gamma"][ch].double(), s["beta"][ch].double()
        fs = s["film"][:, None, ch].double() if case["film"] else 1.0
        if case["op"] == NORM:
            x = s["x"][:, :, ch].double()
            m = x.mean((1, 2), keepdim=True)
            r = 1 / torch.sqrt(((x - m) ** 2).mean((1, 2), keepdim=True) + EPS)
            a = fs * _exact_act(case["act"], (x - m) * r * ga + be)[0]
            out["y"].append(a + s["film"][:, None, C + j * w:C + j * w + w].double() if case["film"] else a)
            out["mean"].append(m[:, :, 0])
            out["rstd"].append(r[:, :, 0])
            continue
        r = s["rstd"][:, j].double()[:, None, None]
        h = (values[:, :, ch] - s["mean"][:, j].double()[:, None, None]) * r
        a, da = _exact_act(case["act"], h * ga + be)
        dy = s["dy"][:, :, ch].double()
        dz = dy * fs * da
        dh = dz * ga
        out["dx"].append(r * (dh - dh.mean((1, 2), keepdim=True) - h * (dh * h).mean((1, 2), keepdim=True)))
        out["dgamma"].append((dz * h).sum((0, 1)))
        out["dbeta"].append(dz.sum((0, 1)))
        out["ds"].append((dy * a).sum(1))
        out["db"].append(dy.sum(1))
    if case["op"] == NORM:
        got = dict(y=torch.cat(out["y"], 2), mean=torch.cat(out["mean"], 1), rstd=torch.cat(out["rstd"], 1))
        if case["saved"]:
            got.update(saved_x=_exact_copy(s["x"].reshape(N * L, C)), saved_y=None)      # (of y as it is rounded)
        return got
    got = dict(dx=torch.cat(out["dx"], 2), dgamma=torch.cat(out["dgamma"]), dbeta=torch.cat(out["dbeta"]))
    return dict(got, dfilm=torch.cat(out["ds"] + out["db"], 1)) if case["film"] else got
