"""Problems and double-precision references for the products with bit-packed weights (textbook definitions only)."""
import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # of a rounding, relative to the value


def pack_rows(codes, bits):
    """The little-endian bit stream of every row as 32-bit words."""
    rows, d = codes.shape
    stream = np.unpackbits(codes.astype(np.uint8).reshape(-1, 1), axis=1, bitorder="little")[:, :bits].reshape(rows, d * bits)
    return np.packbits(stream, axis=1, bitorder="little").view("<i4")


def problem(seed, n_tok, rows, d, bits, group, dtype, n_adapters=0, rank=0, starts=None, ids=None):
    """CPU tensors of a case; starts / ids describe the requests."""
    r = np.random.default_rng(seed)
    n_g = d // group if group else 1
    t = torch.from_numpy
    p = dict(n_tok=n_tok, rows=rows, d=d, bits=bits, group=group, dtype=dtype)
    codes = r.integers(0, 1 << bits, (rows, d))
    p["scales"] = t((0.5 + r.random((rows, n_g))).astype(np.float32) * 0.1 / 2 ** bits)
    p["zeros"] = t(r.integers(0, 1 << bits, (rows, n_g)).astype(np.int32))
    p["packed"] = t(pack_rows(codes, bits).copy())
    zz = np.repeat(p["zeros"].numpy(), d // n_g, 1)
    p["Q"] = t((codes - zz) * np.repeat(p["scales"].numpy().astype(np.float64), d // n_g, 1))
    p["x"] = t(r.standard_normal((n_tok, d)).astype(np.float32) * np.exp(0.5 * r.standard_normal((n_tok, 1))).astype(np.float32)).to(dtype)
    p["dy"] = t(r.standard_normal((n_tok, rows)).astype(np.float32)).to(dtype)
    if n_adapters:
        p["A"] = t(r.standard_normal((n_adapters, rank, d)).astype(np.float32) / d ** 0.5).to(dtype)
        p["B"] = t(r.standard_normal((n_adapters, rank, rows)).astype(np.float32) * 0.1).to(dtype)
        p["scale"] = t((0.5 + r.random(n_adapters)).astype(np.float32))
        p["starts"] = torch.tensor(starts, dtype=torch.int32)
        p["ids"] = torch.tensor(ids, dtype=torch.int32)
    return p


def owners(p):
    """The adapter of every token, -1 for none."""
    out = torch.full((p["n_tok"],), -1, dtype=torch.int64)
    if "ids" in p:
        s = p["starts"].tolist()
        for j, i in enumerate(p["ids"].tolist()):
            if 0 <= i < p["scale"].shape[0]:
                out[s[j]:s[j + 1]] = i
    return out


def forward64(p):
    """(y, xa, bound): in double, and the bound on the error of y computed in float sums and rounded once."""
    x, Q = p["x"].double(), p["Q"]
    y, size = x @ Q.T, x.abs() @ Q.abs().T
    xa = None
    if "ids" in p:
        own = owners(p)
        rank = p["A"].shape[1]
        xa = torch.zeros((p["n_tok"], rank), dtype=torch.float64)
        for i in range(p["A"].shape[0]):
            m = own == i
            A, B, c = p["A"][i].double(), p["B"][i].double(), p["scale"][i].double()
            xa[m] = x[m] @ A.T
            y[m] += c * (xa[m] @ B)
            size[m] += c * ((x[m].abs() @ A.abs().T) @ B.abs())
    return y, xa, sum_bound(p["d"], size, p["dtype"]) + HALF_STEP[p["dtype"]] * y.abs()


def sum_bound(n, size, dtype):
    """Float sums of n products whose magnitudes add up to `size`: at most n 2^-23 of it, and in bf16 two pieces of bf16 may stand
    for a float between two products (2^-16)."""
    return ((n + 64) * 2.0 ** -23 + (2.0 ** -16 if dtype == torch.bfloat16 else 0.0)) * size


def backward64(p, x=None, xa=None):
    """dict name -> (value, bound) of dx, dA, dB in double."""
    dy, Q, dtype = p["dy"].double(), p["Q"], p["dtype"]
    dx, size = dy @ Q, dy.abs() @ Q.abs()
    # in bf16 the weights are rounded to bf16 on the way
    weights = (HALF_STEP[dtype] * 1.01 if dtype == torch.bfloat16 else 0.0) * size
    res = {}
    if "ids" in p:
        own = owners(p)
        x = p["x"].double() if x is None else x.double()
        dA, dB = torch.zeros(p["A"].shape, dtype=torch.float64), torch.zeros(p["B"].shape, dtype=torch.float64)
        sA, sB = dA.clone(), dB.clone()
        for i in range(p["A"].shape[0]):
            m = own == i
            A, B, c = p["A"][i].double(), p["B"][i].double(), p["scale"][i].double()
            u, us = c * (dy[m] @ B.T), c * (dy[m].abs() @ B.abs().T)
            dx[m] += u @ A
            size[m] += us @ A.abs()
            dA[i], sA[i] = u.T @ x[m], us.T @ x[m].abs()
            dB[i], sB[i] = c * (xa[m].double().T @ dy[m]), c * (xa[m].double().abs().T @ dy[m].abs())
        n = p["n_tok"] + p["rows"]
        res["dA"], res["dB"] = (dA, (n + 64) * 2.0 ** -23 * sA), (dB, (n + 64) * 2.0 ** -23 * sB)
    res["dx"] = (dx, sum_bound(p["rows"], size, dtype) + weights + HALF_STEP[dtype] * 1.01 * (dx.abs() + weights))
    return res


def on_gpu(tb, p):
    """(weight, adapters or None) on the current device."""
    c = lambda n: p[n].cuda()  # noqa: E731
    w = tb.packed_weight(c("packed"), c("scales"), c("zeros"), p["d"], p["bits"], p["group"])
    a = tb.adapters(c("A"), c("B"), c("scale"), c("starts"), c("ids")) if "ids" in p else None
    return w, a


def near(got, want, bound, what=""):
    """Every value within its bound, and what is not a number in the same places."""
    got = got.cpu().double()
    assert got.shape == want.shape, what
    off = (got - want).abs() - bound
    assert not torch.isnan(got).any(), what
    assert off.max().item() <= 0.0, (what, off.max().item(), int(off.argmax()))


def norm_off(got, want):
    return float((got.cpu().double() - want).norm() / want.norm().clamp(min=1e-300))


def eight_bits(x):
    """(codes, scales) of the 8-bit form, quotients in double."""
    n, d = x.shape
    codes, scales = np.zeros((n, d), np.int8), np.zeros((n, -(-d // 128)), np.float32)
    v = x.float().numpy()
    for g in range(scales.shape[1]):
        part = v[:, 128 * g:128 * (g + 1)]
        s = np.abs(part).max(1) / np.float32(127.0)
        scales[:, g] = s
        with np.errstate(divide="ignore", invalid="ignore"):
            q = np.where(s[:, None] > 0, np.rint(part.astype(np.float64) / s[:, None].astype(np.float64)), 0.0)
        codes[:, 128 * g:128 * (g + 1)] = np.clip(q, -127, 127)
    return codes, scales
