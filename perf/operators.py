"""Measured cases of the products with bit-packed weights: what a program that serves or fine-tunes a quantized layer calls.

Five kinds of work, each through the functions of the package where `own` is true, in elementary torch operations where it is false:

  linear      y = x Q^T, Q = diag(s)(W_int - z) held as a packed bit stream with float scales and integer zero-points
  adapters    the same with low-rank adapters of many requests beside it: y_t += c_i (x_t A_i^T) B_i for the tokens t of a request
              with adapter i
  backward    the gradients of that: dx = dy Q + c_i (dy B_i^T) A_i, dA_i = sum_t c_i (dy_t B_i^T)^T x_t and dB_i = sum_t
              c_i (x_t A_i^T)^T dy_t, with x in full or held in 8 bits
  step        one training step of such a layer: forward, the input kept in 8 bits, backward from what was kept
  checkpoint  activations to 8 bits with one scale for every token and 128 columns, and back

An adapter's two matrices are [rank][d_in] and [rank][d_out].  Requests are runs of tokens: request j has the tokens
starts[j] .. starts[j + 1] - 1 and adapter ids[j], or none where that is negative.
"""
import torch

own = False

DEV = "cuda:0"
CKPT = 128  # columns of a token that share a scale in 8 bits


def listed():
    return [
        # One token through a 4096-wide query projection in INT4: the smallest call of a decoding loop, all latency.
        dict(name="linear_1tok_4096_w4", kind="linear", tokens=1, rows=4096, d=4096, bits=4, gq=128, dtype="bf16"),
        # One token through an 8192-wide projection in INT2: 16 MB of codes, bound by reading them.
        dict(name="linear_1tok_8192_w2", kind="linear", tokens=1, rows=8192, d=8192, bits=2, gq=128, dtype="bf16"),
        # A prompt of 4096 tokens through the same: a large matrix product whose weights are decoded on the way.
        dict(name="linear_4096tok_8192_w2", kind="linear", tokens=4096, rows=8192, d=8192, bits=2, gq=128, dtype="bf16"),
        # Float activations, an odd number of tokens, 3-bit codes that straddle words, narrow groups.
        dict(name="linear_f32_77tok_1920_w3", kind="linear", tokens=77, rows=1152, d=1920, bits=3, gq=64, dtype="f32"),
        # A decoding step of 64 requests, one token each, over 48 adapters of rank 16.
        dict(name="adapters_64req_4096_w4", kind="adapters", tokens=64, rows=4096, d=4096, bits=4, gq=128, dtype="bf16",
             requests=64, n_adapters=48, rank=16),
        # Few requests through a key projection of grouped-query attention: few rows, a long contraction.
        dict(name="adapters_8req_1024x8192_w2", kind="adapters", tokens=8, rows=1024, d=8192, bits=2, gq=128, dtype="bf16",
             requests=8, n_adapters=8, rank=8),
        # Prompts of ragged lengths, some requests empty or without an adapter, 3-bit codes.
        dict(name="adapters_1999tok_4096_w3", kind="adapters", tokens=1999, rows=4096, d=4096, bits=3, gq=128, dtype="bf16",
             requests=23, n_adapters=9, rank=32),
        # Fine-tuning one adapter beside a 4-bit projection: 8192 tokens a step, the input kept in bf16.
        dict(name="backward_8192tok_4096_w4", kind="backward", tokens=8192, rows=4096, d=4096, bits=4, gq=128, dtype="bf16",
             requests=1, n_adapters=1, rank=16, ckpt=False),
        # Three adapters of rank 64 trained together on an 8192-wide 2-bit projection, the input kept in 8 bits.
        dict(name="backward_4099tok_8192_w2_ckpt", kind="backward", tokens=4099, rows=8192, d=8192, bits=2, gq=128,
             dtype="bf16", requests=5, n_adapters=3, rank=64, ckpt=True),
        # A whole small step of an odd layer: 13 heads, 301 tokens, one scale per row.
        dict(name="step_301tok_1664_w4", kind="step", tokens=301, rows=1664, d=1664, bits=4, gq=0, dtype="bf16", requests=4,
             n_adapters=2, rank=8),
        # The activations of a long batch to 8 bits and back, bound by memory.
        dict(name="checkpoint_16384x8192", kind="checkpoint", tokens=16384, d=8192, dtype="bf16"),
        # A short ragged batch: latency again.
        dict(name="checkpoint_33x4096", kind="checkpoint", tokens=33, d=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, spread over the logarithm."""
    v = lo * (hi / lo) ** rng.random()
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "adapters", "adapters", "adapters", "backward", "backward", "step", "checkpoint"])
    dtype = rng.choice(["bf16"] * 5 + ["f32"])
    d = _log(rng, 256, 8192, rng.choice([128, 128, 128, 32]))
    tokens = _log(rng, 1, 4096) if kind in ("linear", "adapters") else _log(rng, 16, 4096)
    if kind == "checkpoint":
        return dict(kind=kind, tokens=_log(rng, 1, 16384), d=d, dtype=dtype)
    rows = _log(rng, 256, 8192, rng.choice([128, 128, 64, 8]))
    if dtype == "f32":
        tokens = min(tokens, 1024)
    c = dict(kind=kind, tokens=tokens, rows=rows, d=d, bits=rng.choice([2, 2, 3, 3, 4, 4, 5, 6, 7, 8]),
             gq=rng.choice([0] + [q for q in (32, 64, 128, 128, 256) if d % q == 0]), dtype=dtype)
    if kind != "linear":
        c |= dict(requests=min(tokens, _log(rng, 1, 128)) if kind == "adapters" else rng.randint(1, 8),
                  n_adapters=rng.randint(1, 64) if kind == "adapters" else rng.randint(1, 4),
                  rank=rng.choice([8, 16, 16, 32, 64, 128]))
    if kind == "backward":
        c["ckpt"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------------------------------ inputs

def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _activations(g, n_tok, d, dtype):
    """Heavy-tailed activations: log-normal token scale, 1 % of the channels x 20."""
    sigma = torch.ones(d, device=DEV)
    sigma[torch.randperm(d, generator=g, device=DEV)[:max(1, d // 100)]] = 20.0
    x = torch.randn((n_tok, d), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((n_tok, 1), generator=g, device=DEV))
    return (x * sigma).to(dtype)


def _pack(codes, bits):
    """The little-endian bit stream of every row as 32-bit words: 32 codes take `bits` words."""
    rows, d = codes.shape
    out = []
    for r in range(0, rows, 2048):
        v = codes[r:r + 2048].to(torch.int32)
        stream = torch.stack([(v >> b) & 1 for b in range(bits)], -1).reshape(v.shape[0], d * bits // 32, 32)
        words = (stream.to(torch.int64) << torch.arange(32, device=DEV)).sum(-1)
        out.append(torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32))
    return torch.cat(out).contiguous()


def _weight(g, c):
    rows, d, bits = c["rows"], c["d"], c["bits"]
    groups = 1 if c["gq"] == 0 else d // c["gq"]
    codes = torch.randn((rows, d), generator=g, device=DEV) * 2 ** bits / 6 + (2 ** bits - 1) / 2
    codes = codes.round().clamp(0, 2 ** bits - 1).to(torch.uint8)
    scales = (0.5 + torch.rand((rows, groups), generator=g, device=DEV)) * 0.08 / 2 ** bits
    zeros = (2 ** (bits - 1) + torch.randint(-1, 2, (rows, groups), generator=g, device=DEV)).clamp(0, 2 ** bits - 1).to(torch.int32)
    return dict(packed=_pack(codes, bits), scales=scales, zeros=zeros)


def _requests(g, c):
    """Ragged runs of tokens; with four requests and more one in eight has no adapter and, where there are fewer requests
    than tokens, the second is empty."""
    n, t = c["requests"], c["tokens"]
    if n == t:
        starts = torch.arange(n + 1, device=DEV, dtype=torch.int32)
    else:
        cuts = torch.sort(torch.randint(0, t + 1, (n - 1,), generator=g, device=DEV))[0].to(torch.int32)
        starts = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), t)])
        if n >= 4:
            starts[2] = starts[1]
    ids = torch.randint(0, c["n_adapters"], (n,), generator=g, device=DEV).to(torch.int32)
    if n >= 4:
        ids[7::8] = -1
    return starts, ids


def _adapters(g, c):
    k, r = c["n_adapters"], c["rank"]
    starts, ids = _requests(g, c)
    A = (torch.randn((k, r, c["d"]), generator=g, device=DEV) / c["d"] ** 0.5).to(_type(c))
    B = (torch.randn((k, r, c["rows"]), generator=g, device=DEV) * 0.05).to(_type(c))
    scale = 0.5 + torch.rand(k, generator=g, device=DEV)
    return dict(A=A, B=B, scale=scale, starts=starts, ids=ids)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + 29)
    s = dict(case=c, x=_activations(g, c["tokens"], c["d"], _type(c)))
    if c["kind"] == "checkpoint":
        return s
    s |= _weight(g, c)
    if c["kind"] != "linear":
        s |= _adapters(g, c)
    if c["kind"] in ("backward", "step"):
        s["dy"] = _activations(g, c["tokens"], c["rows"], _type(c)) * 0.01
    if c["kind"] == "backward":  # what the forward pass of the training step left
        s["xa"] = _low(s["x"].float(), s["A"].float(), s["starts"], s["ids"])
        if c["ckpt"]:
            s["codes"], s["cscales"] = _to_8_bits(s.pop("x"))
    return s


# ------------------------------------------------------------------------------------------ the plain forms

def _dequantized(s):
    """Q = diag(s)(W_int - z) in float from the packed words."""
    c = s["case"]
    at = torch.arange(c["d"], device=DEV) * c["bits"]
    words = torch.nn.functional.pad(s["packed"], (0, 1)).to(torch.int64) & 0xFFFFFFFF
    pair = words[:, at // 32] | (words[:, at // 32 + 1] << 32)
    codes = (pair >> (at % 32)) & (2 ** c["bits"] - 1)
    n_g = s["scales"].shape[1]
    codes = codes.reshape(c["rows"], n_g, c["d"] // n_g)
    return ((codes - s["zeros"][:, :, None]).float() * s["scales"][:, :, None]).reshape(c["rows"], c["d"])


def _owner(starts, ids, n_tok, n_adapters):
    """[n_tok][n_adapters] in float: 1 where a token belongs to a request with that adapter."""
    t = torch.arange(n_tok, device=DEV, dtype=torch.int32)
    j = torch.searchsorted(starts, t, right=True) - 1
    return (ids[j][:, None] == torch.arange(n_adapters, device=DEV)[None, :]).float()


def _low(x, A, starts, ids):
    """x_t A_i^T for the adapter i of every token t, zero where it has none: [n_tok][rank]."""
    k, r, d = A.shape
    every = (x @ A.reshape(k * r, d).T).reshape(-1, k, r)
    return (every * _owner(starts, ids, x.shape[0], k)[:, :, None]).sum(1)


def _spread(v, owner):
    """[n_tok][rank] to [n_tok][n_adapters * rank], with zeros at the adapters that are not the token's."""
    return (v[:, None, :] * owner[:, :, None]).reshape(v.shape[0], -1)


def _to_8_bits(x):
    """Codes -127 .. 127 and float scales of runs of 128 columns of a token (the last run may be shorter)."""
    n_tok, d = x.shape
    n_g = -(-d // CKPT)
    v = torch.nn.functional.pad(x.float(), (0, n_g * CKPT - d)).reshape(n_tok, n_g, CKPT)
    scale = (v.abs().amax(-1).double() / 127).float()
    codes = (v.double() / scale.double()[:, :, None]).round().nan_to_num(0.0).clamp(-127, 127)
    return codes.reshape(n_tok, -1)[:, :d].to(torch.int8).contiguous(), scale


def _from_8_bits(codes, scale):
    return codes.float() * scale.repeat_interleave(CKPT, 1)[:, :codes.shape[1]]


def _plain_forward(s):
    c, x = s["case"], s["x"].float()
    y = x @ _dequantized(s).T
    if c["kind"] == "linear":
        return y, None
    k, r = c["n_adapters"], c["rank"]
    xa = _low(x, s["A"].float(), s["starts"], s["ids"])
    owner = _owner(s["starts"], s["ids"], c["tokens"], k)
    return y + _spread(xa, owner * s["scale"]) @ s["B"].float().reshape(k * r, -1), xa


def _plain_backward(s, x, xa):
    c, dy = s["case"], s["dy"].float()
    k, r = c["n_adapters"], c["rank"]
    A, B = s["A"].float(), s["B"].float()
    owner = _owner(s["starts"], s["ids"], c["tokens"], k) * s["scale"]
    u = _spread(_low(dy, B, s["starts"], s["ids"]), owner)
    dx = dy @ _dequantized(s) + u @ A.reshape(k * r, -1)
    dA = (u.T @ x).reshape(A.shape)
    dB = (_spread(xa, owner).T @ dy).reshape(B.shape)
    return dict(dx=dx.to(_type(c)), dA=dA, dB=dB)


def _given(y, xa, dtype):
    return dict(y=y.to(dtype)) if xa is None else dict(y=y.to(dtype), xa=xa)


def _plain(s):
    c = s["case"]
    if c["kind"] == "checkpoint":
        codes, scale = _to_8_bits(s["x"])
        return dict(values=_from_8_bits(codes, scale).to(_type(c)), scales=scale)
    if c["kind"] in ("linear", "adapters"):
        return _given(*_plain_forward(s), _type(c))
    if c["kind"] == "backward":
        return _plain_backward(s, _from_8_bits(s["codes"], s["cscales"]) if c["ckpt"] else s["x"].float(), s["xa"])
    y, xa = _plain_forward(s)
    return dict(y=y.to(_type(c)), **_plain_backward(s, _from_8_bits(*_to_8_bits(s["x"])), xa))


# ------------------------------------------------------------------------------------------ one pass

def run(state):
    return _calls(state) if own else _plain(state)


def _calls(s):
    import paper_2602_04929_b200 as tb
    c = s["case"]
    if c["kind"] == "checkpoint":
        codes, scales = tb.tb_checkpoint_pack(s["x"])
        return dict(values=tb.tb_checkpoint_unpack(codes, scales, _type(c)), scales=scales)
    if "handle" not in s:  # a program makes these once beside the tensors: they hold no data of their own
        s["handle"] = (tb.packed_weight(s["packed"], s["scales"], s["zeros"], c["d"], c["bits"], c["gq"]),
                       None if c["kind"] == "linear" else tb.adapters(s["A"], s["B"], s["scale"], s["starts"], s["ids"]))
    w, ad = s["handle"]
    if c["kind"] in ("linear", "adapters"):
        return _given(*tb.tb_packed_linear(w, s["x"], ad), _type(c))
    if c["kind"] == "backward":
        kept = dict(checkpoint=(s["codes"], s["cscales"])) if c["ckpt"] else dict(x=s["x"])
        dx, dA, dB = tb.tb_packed_linear_backward(w, s["dy"], ad, xa=s["xa"], **kept)
        return dict(dx=dx, dA=dA, dB=dB)
    y, xa = tb.tb_packed_linear(w, s["x"], ad)
    kept = tb.tb_checkpoint_pack(s["x"])
    dx, dA, dB = tb.tb_packed_linear_backward(w, s["dy"], ad, xa=xa, checkpoint=kept)
    return dict(y=y, dx=dx, dA=dA, dB=dB)


# ------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    t, d, size = c["tokens"], c["d"], 2 if c["dtype"] == "bf16" else 4
    eight = t * d + 4.0 * t * -(-d // CKPT)
    if c["kind"] == "checkpoint":  # in, codes and scales out, read back, values out
        return {"bytes": 2.0 * size * t * d + 2 * eight, "flops": 4.0 * t * d}
    rows = c["rows"]
    weight = rows * d * c["bits"] / 8 + 8.0 * rows * (1 if c["gq"] == 0 else d // c["gq"])
    product, io = 2.0 * t * rows * d, float(size) * t * (rows + d)
    if c["kind"] == "linear":
        return {"bytes": weight + io, "flops": product}
    used = min(c["n_adapters"], c["requests"]) * c["rank"] * (rows + d)
    low, kept = 2.0 * t * c["rank"] * (rows + d), 4.0 * t * c["rank"]
    forward = {"bytes": weight + io + size * used, "flops": product + low}
    grads = 4.0 * c["n_adapters"] * c["rank"] * (rows + d)
    back = {"bytes": weight + io + size * used + grads + kept, "flops": product + 2 * low}
    if c["kind"] == "adapters":
        return forward
    if c["kind"] == "backward":
        return {"bytes": back["bytes"] + (eight if c["ckpt"] else size * t * d), "flops": back["flops"]}
    return {"bytes": forward["bytes"] + back["bytes"] + 2 * eight + 2 * kept, "flops": forward["flops"] + back["flops"]}


# ------------------------------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    """From the definition, request by request, in double."""
    c, s = case, prepare(case, seed)
    f8 = torch.float64

    def eight(x):  # the scales are floats of the format itself: one rounding of amax / 127
        out, all_scales = torch.empty(x.shape, dtype=f8, device=DEV), []
        for lo in range(0, c["d"], CKPT):
            part = x[:, lo:lo + CKPT].to(f8)
            scale = (part.abs().max(1)[0] / 127.0).float().to(f8)[:, None]
            out[:, lo:lo + CKPT] = torch.where(scale > 0, torch.round(part / scale.clamp(min=1e-300)), 0.0) * scale
            all_scales.append(scale)
        return out, torch.cat(all_scales, 1)

    if c["kind"] == "checkpoint":
        values, scales = eight(s["x"])
        return dict(values=values, scales=scales)
    raw = s["packed"].view(torch.uint8)
    bit = torch.stack([(raw >> i) & 1 for i in range(8)], -1).reshape(c["rows"], c["d"], c["bits"])
    codes = torch.zeros((c["rows"], c["d"]), dtype=f8, device=DEV)
    for i in range(c["bits"]):
        codes += bit[:, :, i].to(f8) * 2.0 ** i
    width = c["d"] if c["gq"] == 0 else c["gq"]
    Q = torch.empty_like(codes)
    for j in range(c["d"] // width):
        cols = slice(j * width, (j + 1) * width)
        Q[:, cols] = s["scales"][:, j:j + 1].to(f8) * (codes[:, cols] - s["zeros"][:, j:j + 1].to(f8))
    del codes, bit
    runs = []
    if c["kind"] != "linear":
        at = s["starts"].tolist()
        runs = [(slice(at[j], at[j + 1]), i) for j, i in enumerate(s["ids"].tolist()) if i >= 0]
        A, B, scale = s["A"].to(f8), s["B"].to(f8), s["scale"].to(f8)
    res = {}
    if c["kind"] != "backward":
        x = s["x"].to(f8)
        y = x @ Q.T
        for tok, i in runs:
            y[tok] += scale[i] * ((x[tok] @ A[i].T) @ B[i])
        res["y"] = y
        if c["kind"] == "adapters":
            res["xa"] = torch.zeros((c["tokens"], c["rank"]), dtype=f8, device=DEV)
            for tok, i in runs:
                res["xa"][tok] = x[tok] @ A[i].T
    if c["kind"] in ("backward", "step"):
        dy = s["dy"].to(f8)
        if c["kind"] == "step":
            xa = torch.zeros((c["tokens"], c["rank"]), dtype=f8, device=DEV)
            for tok, i in runs:
                xa[tok] = x[tok] @ A[i].T
            x = eight(s["x"])[0]
        else:
            xa = s["xa"].to(f8)
            x = s["codes"].to(f8) * s["cscales"].to(f8).repeat_interleave(CKPT, 1)[:, :c["d"]] if c["ckpt"] else s["x"].to(f8)
        dx, dA, dB = dy @ Q, torch.zeros_like(A), torch.zeros_like(B)
        for tok, i in runs:
            u = scale[i] * (dy[tok] @ B[i].T)
            dx[tok] += u @ A[i]
            dA[i] += u.T @ x[tok]
            dB[i] += scale[i] * (xa[tok].T @ dy[tok])
        res |= dict(dx=dx, dA=dA, dB=dB)
    return res
