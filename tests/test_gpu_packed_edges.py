"""The products with bit-packed weights where they could go wrong: no tokens, the widest rows, the largest activations, zero-points
beyond the codes, infinities in adapters, and how near the sums come to those in 64 bits."""
import numpy as np
import pytest
import torch

import packed_util as pu

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _tb():
    import paper_2602_04929_b200 as tb
    return tb


@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward_without_tokens(dtype):
    """An empty batch has an empty dx, whether or not adapters and a kept input come with it."""
    tb = _tb()
    p = pu.problem(1, 0, 64, 96, 3, 32, dtype, 2, 8, [0, 0], [1])
    w, a = pu.on_gpu(tb, p)
    for ad in (None, a):
        dx, dA, dB = tb.tb_packed_linear_backward(w, p["dy"].cuda(), ad)
        assert dx.shape == (0, 96) and dx.dtype == dtype and dA is None and dB is None


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_widest_rows(dtype):
    """2^24 columns of the result, both directions: 256 tokens of them are 2^32 values.  The last of a tile's tokens lie 255 rows from its
    first, past 2^31 values; they and others against double precision."""
    tb = _tb()
    n_tok, wide = (256, 1 << 24) if dtype == BF else (100, 1 << 24)
    g = torch.Generator(device="cuda").manual_seed(8)
    ints = lambda lo, hi, shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    looked_at = [0, n_tok // 2 - 1, n_tok // 2, n_tok - 1]

    def weights(rows, d):
        words = torch.randint(-1 << 31, 1 << 31, (rows, d // 16), generator=g, device="cuda").to(torch.int32)
        w = tb.packed_weight(words, torch.rand((rows, 1), generator=g, device="cuda") + 0.5, ints(0, 4, (rows, 1)), d, 2)
        codes = (words.unsqueeze(-1) >> torch.arange(0, 32, 2, device="cuda", dtype=torch.int32)) & 3
        return w, (codes.view(rows, d).double() - w.tensors[2]) * w.tensors[1].double()

    def check(got, v, k, weights=0.0):
        """Float sums, the result's rounding, and a rounding of every weight by `weights` of it: the last two come one after the other,
        each half a step (2^-8 in bf16) at most."""
        for t in looked_at:
            at = v[t].double()
            want, size = at @ k, at.abs() @ k.abs()
            off = (got[t].double() - want).abs()
            bound = pu.sum_bound(k.shape[0], size, dtype) + weights * size + 1.01 * pu.HALF_STEP[dtype] * (want.abs() + weights * size)
            assert (off <= bound).all(), t
            del want, size, off, bound

    # dx of 8 rows, 2 bits
    w, Q = weights(8, wide)
    dy = torch.randn((n_tok, 8), generator=g, device="cuda").to(dtype)
    dx, _, _ = tb.tb_packed_linear_backward(w, dy)
    assert tb.tb_device_error_flag() == 0
    check(dx, dy, Q, pu.HALF_STEP[BF] if dtype == BF else 0.0)
    del dx, Q, w
    # y of 2^24 rows
    w, Q = weights(wide, 32)
    x = torch.randn((n_tok, 32), generator=g, device="cuda").to(dtype)
    y, _ = tb.tb_packed_linear(w, x)
    assert tb.tb_device_error_flag() == 0
    check(y, x, Q.T)


def _within_one(p):
    """The problem with codes of two bits and zero-points of 1 whose differences are -1, 0 and 1."""
    codes = np.random.default_rng(6).integers(0, 3, (p["rows"], p["d"]))
    p["packed"], p["zeros"] = torch.from_numpy(pu.pack_rows(codes, 2).copy()), torch.ones_like(p["zeros"])
    p["Q"] = torch.from_numpy(codes - 1).double() * p["scales"].double().repeat_interleave(p["group"], 1)
    return p


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("n_tok", [3, 40, 97, 200, 1400])
def test_the_largest_activations(n_tok, group, dtype):
    """The largest finite values, where no sum of x (c - z) leaves the range of floats (|c - z| <= 1 here): those of y and dx are finite,
    and right.  3.3953e38 lies between the largest bf16 and what rounds to infinity."""
    tb = _tb()
    p = _within_one(pu.problem(5, n_tok, 264, 256, 2, group, dtype))
    top = torch.finfo(dtype).max
    for t, v in ((0, top), (1, -top), (2, 3.3953e38 if dtype == F32 else -top)):
        p["x"][t, 17 + t], p["dy"][t, 30 + t] = v, v
    w, _ = pu.on_gpu(tb, p)
    y, _ = tb.tb_packed_linear(w, p["x"].cuda())
    want, _, bound = pu.forward64(p)
    pu.near(y, want, bound, "y")
    dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    pu.near(dx, *pu.backward64(p)["dx"], "dx")
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("dtype,n_tok", [(BF, 600), (F32, 40), (F32, 200)])
@pytest.mark.parametrize("rank", [8, 40])
def test_the_largest_sums_of_the_narrow_product(dtype, n_tok, rank):
    """x A^T next to the largest float (3.3995e38 rounds to infinity in bf16), met by small entries of B and of dy: finite outputs and
    gradients."""
    tb = _tb()
    p = _within_one(pu.problem(3, n_tok, 520, 256, 2, 128, dtype, 1, rank, [0, n_tok], [0]))
    p["A"].zero_(), p["B"].mul_(1e-3), p["scale"].fill_(1.0)
    p["A"][0, :, 7:9] = 1.0
    p["x"][:4] *= 2.0 ** -100
    p["x"][:4, 7] = torch.tensor([3.0e38, 3.3895314e38, -3.3895314e38, 3.3895314e38]).to(dtype)
    p["x"][3, 8] = 1e36
    p["scales"], p["Q"] = p["scales"] * 2.0 ** -20, p["Q"] * 2.0 ** -20       # the product itself stays far below the adapters' share
    w, a = pu.on_gpu(tb, p)
    y, xa = tb.tb_packed_linear(w, p["x"].cuda(), a)
    want, xa64, bound = pu.forward64(p)
    pu.near(xa[:4], xa64[:4], 2.0 ** -22 * xa64[:4].abs(), "xa")
    pu.near(y, want, bound, "y")
    xa = xa.clone()
    xa[0], xa[2] = 3.3953e38, -3.4028e38
    p["dy"] = p["dy"] * 2.0 ** -30
    out = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, x=p["x"].cuda(), xa=xa)
    ref = pu.backward64(p, None, xa.cpu())
    for got, name in zip(out, ("dx", "dA", "dB")):
        pu.near(got, *ref[name], name)


def _with_zero_points(p, z):
    d = p["d"]
    wide = lambda v: v.double().repeat_interleave(d // v.shape[1], 1)  # noqa: E731
    return dict(p, zeros=z, Q=p["Q"] + wide(p["zeros"].long() - z.long()) * wide(p["scales"]))


@pytest.mark.parametrize("bits", range(2, 9))
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_tok", [5, 24, 97, 1100])
def test_zero_points_wherever_their_differences_are_exact(bits, dtype, n_tok):
    """Every zero-point whose differences to all codes lie within 256: the products have nothing but float sums and one rounding, on
    both sides of every rule that chooses a kernel."""
    tb = _tb()
    p = pu.problem(bits, n_tok, 264, 256, bits, 32 if bits % 2 else 128, dtype)
    g = torch.Generator().manual_seed(bits)
    z = torch.randint((1 << bits) - 257, 257, p["zeros"].shape, generator=g, dtype=torch.int32)
    z[::3] = torch.randint(129, 257, z[::3].shape, generator=g, dtype=torch.int32)
    p = _with_zero_points(p, z)
    w, _ = pu.on_gpu(tb, p)
    want, _, bound = pu.forward64(p)
    pu.near(tb.tb_packed_linear(w, p["x"].cuda())[0], want, bound, "y")
    pu.near(tb.tb_packed_linear_backward(w, p["dy"].cuda())[0], *pu.backward64(p)["dx"], "dx")


@pytest.mark.parametrize("bits", [2, 3, 4, 7, 8])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_tok", [5, 97, 1100])
def test_zero_points_far_away(bits, dtype, n_tok):
    """Differences beyond 256 are rounded to bf16: of a code and the zero-point's first piece, of that and the second, and with two bits of
    the first piece less 120: two or three roundings, each off by 2^-8 of the difference at most (and a float's, 2^-23, where the zero-point
    has more than 24 bits)."""
    tb = _tb()
    p = pu.problem(bits, n_tok, 264, 256, bits, 128, dtype)
    g = torch.Generator().manual_seed(bits)
    far = torch.cat([torch.randint(257, 5000, (100, 2), generator=g), torch.randint(-5000, -257, (100, 2), generator=g),
                     torch.tensor([[5000001, -5000001], [8388607, -8388609], [16777217, -16777219], [2147483647, -2147483648]])])
    z = p["zeros"].clone()
    z[:204] = far.to(torch.int32)
    p = _with_zero_points(p, z)
    near = p["scales"] / (1 + 0.01 * z.double().abs()).float()    # so that no row drowns the others
    p["Q"] = p["Q"] * (near.double() / p["scales"].double()).repeat_interleave(128, 1)
    p["scales"] = near
    w, _ = pu.on_gpu(tb, p)
    far = (3.03 if bits == 2 else 2.02) * 2.0 ** -8
    size = p["x"].double().abs() @ p["Q"].abs().T
    want, _, bound = pu.forward64(p)
    pu.near(tb.tb_packed_linear(w, p["x"].cuda())[0], want, bound + far * size, "y")
    want, bound = pu.backward64(p)["dx"]
    pu.near(tb.tb_packed_linear_backward(w, p["dy"].cuda())[0], want, bound + far * (p["dy"].double().abs() @ p["Q"].abs()), "dx")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bits,group", [(2, 128), (4, 32), (5, 128), (7, 128)])
@pytest.mark.parametrize("n_tok", [3, 20, 1100])
def test_infinite_activations_beside_zero_points_of_every_kind(bits, group, n_tok, dtype):
    """Rows with zero-points among the codes and rows with others side by side: an infinite activation comes to what the formula says in all."""
    tb = _tb()
    p = pu.problem(bits, n_tok, 264, 256, bits, group, dtype)
    g = torch.Generator().manual_seed(bits)
    z = p["zeros"].clone()
    z[::3] = torch.randint(129, 257, z[::3].shape, generator=g, dtype=torch.int32)
    z[1::9] = torch.randint(-900, -384, z[1::9].shape, generator=g, dtype=torch.int32)
    p = _with_zero_points(p, z)
    clean = p["x"].clone()
    p["x"][0, 17], p["x"][1, 200] = float("inf"), float("-inf")
    w, _ = pu.on_gpu(tb, p)
    y = tb.tb_packed_linear(w, p["x"].cuda())[0].cpu().double()
    for t, j in ((0, 17), (1, 200)):
        k = p["Q"][:, j]
        assert torch.isnan(y[t][k == 0]).all() and torch.equal(y[t][k != 0], p["x"][t, j].double() * k[k != 0])
    want, _, bound = pu.forward64(dict(p, x=clean))
    pu.near(y[2:], want[2:], bound[2:] + 2.02 * 2.0 ** -8 * (clean.double().abs() @ p["Q"].abs().T)[2:], "y")


@pytest.mark.parametrize("rank", [16, 64, 128])
@pytest.mark.parametrize("n_req", [3, 600])
@pytest.mark.parametrize("n_tok,rows,d", [(600, 520, 256), (2600, 264, 512)])
def test_what_is_not_finite_in_tiles(rank, n_req, n_tok, rows, d):
    """More than 2^18 results, so tiles, with the adapters in stages of their own (few requests, backward the larger shape) or joined to float
    sums: an infinity or what is no number stays with its token or its adapter's requests, both ways, and an infinity that meets an
    infinity is one."""
    tb = _tb()
    starts = [n_tok * k // n_req for k in range(n_req + 1)]
    ids = [1, 0, 1] if n_req == 3 else [k % 3 - 1 for k in range(n_req)]
    p = pu.problem(rank, n_tok, rows, d, 4, 128, BF, 3, rank, starts, ids)
    own = pu.owners(p)
    mine, others = (own == 0).nonzero().flatten().tolist(), own != 0
    nan_tok, inf_tok = mine[1], mine[2]
    # token inf_tok has an infinity at input column k (y's column 40) or at row j of dy (dx's column 50): all its terms are positive infinities
    k, j = int((p["Q"][40, :50] > 0).nonzero()[0]), int((p["Q"][:40, 50] > 0).nonzero()[0])
    g = torch.Generator().manual_seed(rank)
    p["B"][0, :, 40] = p["A"][0, :, k].sign() * (0.1 + torch.rand(rank, generator=g)).to(BF)
    p["A"][0, :, 50] = p["B"][0, :, j].sign() * (0.1 + torch.rand(rank, generator=g)).to(BF)
    p["A"][2] = float("nan")                       # no request has this one
    clean = {n: p[n].clone() for n in ("x", "dy", "A", "B")}
    p["x"][nan_tok, 200], p["x"][inf_tok, k] = float("nan"), float("inf")
    p["dy"][nan_tok, 5], p["dy"][inf_tok, j] = float("nan"), float("inf")
    p["B"][0, 3, 40] = float("inf") * p["B"][0, 3, 40].sign()
    w, a = pu.on_gpu(tb, p)
    y, xa = (v.cpu() for v in tb.tb_packed_linear(w, p["x"].cuda(), a))
    good = dict(p, **clean)
    want, xa64, bound = pu.forward64(good)
    fine = torch.ones(n_tok, dtype=torch.bool)
    fine[[nan_tok, inf_tok]] = False
    cols = torch.ones(rows, dtype=torch.bool)
    cols[40] = False
    pu.near(y[fine][:, cols], want[fine][:, cols], bound[fine][:, cols], "y")
    pu.near(y[fine & others], want[fine & others], bound[fine & others], "y of other requests")
    assert not torch.isfinite(y[~others][:, 40]).any() and torch.isnan(y[nan_tok]).all()
    assert torch.isinf(xa[inf_tok]).all() and torch.isnan(xa[nan_tok]).all() and torch.isfinite(xa[fine]).all()
    assert y[inf_tok, 40] == float("inf")
    one = mine[5]                                  # a finite token of the request: the sign is that of its low value
    assert y[one, 40] == float("inf") * (xa64[one, 3] * p["B"][0, 3, 40].double()).sign()
    # backward, with an infinity in A
    q = dict(good, dy=p["dy"], A=clean["A"].clone())
    q["A"][0, 2, 50] = float("inf") * q["A"][0, 2, 50].sign()
    w, a = pu.on_gpu(tb, q)
    dx, dA, dB = (v.cpu() for v in tb.tb_packed_linear_backward(w, q["dy"].cuda(), a, x=good["x"].cuda(), xa=xa64.float().cuda()))
    ref = pu.backward64(good, None, xa64.float())
    cols = torch.ones(d, dtype=torch.bool)
    cols[50] = False
    pu.near(dx[fine][:, cols], ref["dx"][0][fine][:, cols], ref["dx"][1][fine][:, cols], "dx")
    pu.near(dx[fine & others], ref["dx"][0][fine & others], ref["dx"][1][fine & others], "dx of other requests")
    assert not torch.isfinite(dx[~others][:, 50]).any() and torch.isnan(dx[nan_tok]).all()
    assert dx[inf_tok, 50] == float("inf")
    for got, name in ((dA, "dA"), (dB, "dB")):
        pu.near(got[1], ref[name][0][1], ref[name][1][1], name)
        assert not got[2].any()
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("rows,d,bits,group,n_tok", [(1032, 544, 4, 32, 70), (2056, 1024, 2, 128, 300), (4104, 256, 8, 0, 40), (520, 1152, 7, 384, 700), (8, 160, 3, 32, 5),
                                                     (72, 160, 5, 32, 33), (200, 128, 6, 0, 1100)])
def test_input_gradient_with_all_of_the_weights(rows, d, bits, group, n_tok):
    """dx is off by float sums, by 2^-13.9 of every weight at most (a second bf16 piece of up to 2^-6.9 of it, off by 2^-8 of itself, twice where
    codes have more than four bits) and by its own rounding.  That rounding alone is 1.66e-3 in the norm (2^-8 / sqrt 3 at the power of two,
    times the mean of 1 / m^2 over mantissas m, whose root is 0.74); weights rounded to bf16 would add as much again."""
    tb = _tb()
    p = pu.problem(rows, n_tok, rows, d, bits, group, BF)
    w, _ = pu.on_gpu(tb, p)
    dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    dy, Q = p["dy"].double(), p["Q"]
    want, size = dy @ Q, dy.abs() @ Q.abs()
    weights = ((rows + 64) * 2.0 ** -23 + 2.0 ** (-14.8 if bits <= 4 else -13.9)) * size
    pu.near(dx, want, weights + pu.HALF_STEP[BF] * (want.abs() + weights), "dx")
    if dx.numel() > 10000:
        assert pu.norm_off(dx, want) <= 2.0 ** -9
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("bits,group", [(2, 128), (4, 32), (7, 0)])
@pytest.mark.parametrize("n_tok", [3, 300])
def test_an_infinite_gradient_meets_the_weights(bits, group, n_tok):
    """dy of infinity gives what the formula says, both pieces of a weight having its sign: an infinity of the weight's sign, and what is no
    number where the weight is 0."""
    tb = _tb()
    p = pu.problem(bits, n_tok, 136, 256, bits, group, BF)
    clean = p["dy"].clone()
    p["dy"][0, 30], p["dy"][1, 135], p["dy"][2, 7] = float("inf"), float("-inf"), float("nan")
    w, _ = pu.on_gpu(tb, p)
    dx = tb.tb_packed_linear_backward(w, p["dy"].cuda())[0].cpu().double()
    for t, j in ((0, 30), (1, 135)):
        k = p["Q"][j]
        assert torch.isnan(dx[t][k == 0]).all() and torch.equal(dx[t][k != 0], p["dy"][t, j].double() * k[k != 0])
    assert torch.isnan(dx[2]).all()
    want, bound = pu.backward64(dict(p, dy=clean))["dx"]
    pu.near(dx[3:], want[3:], bound[3:], "dx") if n_tok > 3 else None


def test_input_gradient_of_many_rows():
    """No accumulation of dx is longer than 2048 rows.  The unit drops bits instead of rounding, so errors go to one side: towards 0, at most 2^-23
    of the sum that a step of 16 rows (of either piece) adds to, which on the way to 2048 rows averages 2/3 of their sum: 2/3 * 256 2^-23 of
    dx, whatever the number of rows.  Its rounding goes to both sides: over eight million values 1.66e-3 comes to 5.7e-7 in the mean, at most
    three times that."""
    tb = _tb()
    n_tok, rows, d = 4099, 32768, 2048
    g = torch.Generator(device="cuda").manual_seed(2)
    words = torch.randint(-1 << 31, 1 << 31, (rows, d // 8), generator=g, device="cuda").to(torch.int32)
    scales = 0.01 + 0.01 * torch.rand((rows, d // 128), generator=g, device="cuda")
    zeros = torch.randint(0, 16, (rows, d // 128), generator=g, device="cuda", dtype=torch.int32)
    codes = ((words.unsqueeze(-1) >> torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)) & 15).view(rows, d)
    Q = (codes.double() - zeros.repeat_interleave(128, 1)) * scales.double().repeat_interleave(128, 1)
    dy = torch.randn((n_tok, rows), generator=g, device="cuda").to(BF)
    dx, _, _ = tb.tb_packed_linear_backward(tb.packed_weight(words, scales, zeros, d, 4, 128), dy)
    want = dy.double() @ Q
    shift = ((dx.double() - want) * want.sign()).mean() / want.abs().mean()
    assert abs(shift.item()) <= 2 / 3 * 256 * 2.0 ** -23 + 3 * 5.7e-7
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("n_tok,rows,d,bits,group,rank", [(2600, 4104, 512, 4, 128, 24), (5000, 2056, 256, 7, 32, 64), (3000, 6152, 416, 2, 0, 8)])
def test_input_gradient_of_several_accumulations_with_adapters(n_tok, rows, d, bits, group, rank):
    """More than 2048 rows, a last accumulation of a few, the adapters' stages behind them, several tiles for every pair of processors."""
    tb = _tb()
    p = pu.problem(rank, n_tok, rows, d, bits, group, BF, 3, rank, [5, n_tok // 3, n_tok // 2, n_tok - 7], [2, 0, 1])
    w, a = pu.on_gpu(tb, p)
    dy, Q = p["dy"].cuda().double(), p["Q"].cuda()
    want, size = dy @ Q, dy.abs() @ Q.abs()
    for i in range(3):
        m = (pu.owners(p) == i).cuda()
        A, B, c = p["A"][i].cuda().double(), p["B"][i].cuda().double(), p["scale"][i].double().item()
        want[m] += c * (dy[m] @ B.T) @ A
        size[m] += c * (dy[m].abs() @ B.abs().T) @ A.abs()
    for _ in range(3):
        dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a)
        off = (dx.double() - want).abs()
        inner = (pu.sum_bound(rows + rank, 1.0, BF) + 2.0 ** -13.9) * size     # float sums, pieces of the adapters' sums, pieces of the weights
        assert (off <= inner + pu.HALF_STEP[BF] * (want.abs() + inner)).all()
        assert float((dx.double() - want).norm() / want.norm()) <= 2.0 ** -9
        assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("n_tok,d,rank,n_req", [(16, 524288, 16, 2), (2048, 524288, 64, 2), (5000, 65536, 128, 1), (5000, 65536, 48, 3), (300, 100032, 8, 2), (40, 65536, 128, 7),
                                                (2600, 10240, 112, 2), (1300, 33344, 40, 5)])
def test_sums_of_the_narrow_product(n_tok, d, rank, n_req):
    """No accumulation of x A^T is longer than 512 columns, whatever the rank, the width and the kernel.  A step of 16 columns drops at most
    2^-23 of the sum that it adds to, which on the way to 512 columns averages 2/3 of the sum of 512 (it grows like a root): 32 steps.
    Neighbouring sums have nothing to do with one another; the d / 512 additions that join them round to the nearest, to either side,
    2^-24 each at most, so the root of their number in the norm."""
    tb = _tb()
    p = pu.problem(5, 1, 8, 32, 2, 0, BF, 3, rank, [0, 1], [0])
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    w = tb.packed_weight(ints(8, d // 16), torch.ones((8, 1), device="cuda"), ints(8, 1), d, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n_tok, d), generator=g, device="cuda").to(BF)
    A = (torch.randn((3, rank, d), generator=g, device="cuda") / d ** 0.5).to(BF)
    cuts = [n_tok * k // n_req for k in range(n_req + 1)]
    ids = [k % 3 for k in range(n_req)]
    _, xa = tb.tb_packed_linear(w, x, tb.adapters(A, p["B"].cuda(), p["scale"].cuda(), torch.tensor(cuts, dtype=torch.int32).cuda(),
                                                  torch.tensor(ids, dtype=torch.int32).cuda()))
    off, size = 0.0, 0.0
    for j, i in enumerate(ids):
        for t in range(cuts[j], cuts[j + 1], 512):   # some of them, so that the doubles fit
            s = slice(t, min(t + 64, cuts[j + 1]))
            want = x[s].double() @ A[i].double().T
            off, size = off + float((xa[s] - want).square().sum()), size + float(want.square().sum())
    assert (off / size) ** 0.5 <= 2 / 3 * 32 * 2.0 ** -23 + (d / 512) ** 0.5 * 2.0 ** -24
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("n_tok,rows,d,bits,group,rank", [(208, 832, 2688, 4, 128, 128), (40, 136, 384, 4, 128, 8), (300, 1160, 128, 3, 0, 16), (70, 264, 640, 8, 128, 8),
                                                        (1100, 264, 384, 2, 384, 8), (90, 200, 96, 5, 96, 16), (24, 136, 1152, 7, 128, 16), (1, 8, 32, 2, 32, 8), (5, 40, 160, 3, 32, 24)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_lies_behind_the_inputs_is_not_read(n_tok, rows, d, bits, group, rank, dtype):
    """Every input starts where its alignment just allows it and is followed, without a gap, by values that would show: infinite
    or undefined floats, huge integers.  Outputs, gradients of both forms of the input among them, are right, and the same bits
    whichever values follow."""
    tb = _tb()

    def between(v, word, align):
        n = v.numel() * v.element_size()
        room = torch.full((4096 + n // 4 + 4096,), word, dtype=torch.int32, device="cuda").view(torch.uint8)
        to = room[16384 + align:][:n].view(v.dtype).view(v.shape)
        to.copy_(v)
        return to

    p = pu.problem(n_tok + rows, n_tok, rows, d, bits, group, dtype, 2, rank, sorted([0, n_tok // 3, n_tok // 2, n_tok]), [1, 0, 1])
    w0, a0 = pu.on_gpu(tb, p)
    xa64 = pu.forward64(p)[1].float()
    codes0, scales0 = (torch.from_numpy(v).cuda() for v in pu.eight_bits(p["x"]))
    runs = []
    for word in (0x7f807f80, 0x7fc07fc0, 0x01010101):       # infinities, no numbers, small numbers
        w = tb.packed_weight(*(between(v, word, k) for v, k in zip(w0.tensors, (16, 4, 4))), d, bits, group)
        a = tb.adapters(*(between(v, word, k) for v, k in zip(a0.tensors, (16, 16, 4, 4, 4))))
        x, dy, xa, codes = (between(v.cuda(), word, 16) for v in (p["x"], p["dy"], xa64, codes0))
        scales = between(scales0, word, 4)
        out = [*tb.tb_packed_linear(w, x, a), tb.tb_packed_linear(w, x)[0], *tb.tb_checkpoint_pack(x), tb.tb_checkpoint_unpack(codes, scales, dtype)]
        for kept in (dict(x=x), dict(checkpoint=(codes, scales))):
            out += tb.tb_packed_linear_backward(w, dy, a, xa=xa, **kept)
        runs.append(out)
    for other in runs[1:]:
        assert all(torch.equal(u, v) for u, v in zip(runs[0], other))
    y, _, plain, codes, scales, _, *grads = runs[0]
    want, _, bound = pu.forward64(p)
    pu.near(y, want, bound, "y")
    bare = {k: v for k, v in p.items() if k != "ids"}
    want, _, bound = pu.forward64(bare)
    pu.near(plain, want, bound, "plain")
    assert torch.equal(codes, codes0) and torch.equal(scales, scales0)
    x8 = codes0.double().cpu() * scales0.double().cpu().repeat_interleave(128, 1)[:, :d]
    for got, inp in ((grads[:3], None), (grads[3:], x8)):
        ref = pu.backward64(p, inp, xa64)
        for v, name in zip(got, ("dx", "dA", "dB")):
            pu.near(v, *ref[name], name)
    assert tb.tb_device_error_flag() == 0


def test_8_bit_form_of_the_widest_token():
    """A token of 2^31 - 32 values, its last run a short one: counts of runs and columns stay within what holds them."""
    tb = _tb()
    d = (1 << 31) - 32
    x = torch.empty((1, d), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x.normal_(generator=g)
    codes, scales = tb.tb_checkpoint_pack(x)
    assert scales.shape == (1, 1 << 24)
    back = tb.tb_checkpoint_unpack(codes, scales, BF)
    for s in (slice(0, 4096), slice((1 << 30) - 1024, (1 << 30) + 1024), slice((1 << 31) - 4096, d)):
        part = x[:, s].clone()
        c, k = tb.tb_checkpoint_pack(part)
        assert torch.equal(codes[:, s], c) and torch.equal(scales[:, s.start // 128:-(-s.stop // 128)], k)
        assert torch.equal(back[:, s], tb.tb_checkpoint_unpack(c, k, BF))


def test_outputs_that_lie_over_inputs_are_refused():
    tb = _tb()
    p = pu.problem(1, 40, 64, 64, 4, 0, BF, 2, 64, [0, 40], [0])
    w, a = pu.on_gpu(tb, p)
    x = p["x"].cuda()
    buf = torch.zeros((80, 64), dtype=BF, device="cuda")
    low = torch.zeros((80, 64), device="cuda")
    for call in (lambda: tb.tb_packed_linear(w, x, y=x), lambda: tb.tb_packed_linear(w, buf[20:60], y=buf[:40]),
                 lambda: tb.tb_packed_linear(w, low[:20].view(BF).view(40, 64), a, xa=low[10:50])):
        with pytest.raises(ValueError):
            call()
    y, _ = tb.tb_packed_linear(w, buf[40:], y=buf[:40])        # side by side is fine
    assert y.data_ptr() == buf.data_ptr()


def test_8_bit_scales_are_correctly_rounded():
    """max|x| / 127 for all 2^23 mantissas, at three exponents, one beside what underflows: the bits of a float division."""
    tb = _tb()
    for e in (127, 253, 33):
        top = (torch.arange(1 << 23, device="cuda", dtype=torch.int32) | e << 23).view(torch.float32)
        x = torch.zeros((4096, 2048, 128), device="cuda")
        x[:, :, 5] = top.view(4096, 2048)
        _, scales = tb.tb_checkpoint_pack(x.view(4096, -1))
        want = torch.from_numpy(top.cpu().numpy() / np.float32(127.0))
        assert torch.equal(scales.view(-1).cpu(), want), e
