"""Products with bit-packed weights, adapters beside them and their gradients, element by element against double precision."""
import pytest
import torch

import packed_util as pu

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _tb():
    import paper_2602_04929_b200 as tb
    return tb


def _forward(p, what=""):
    tb = _tb()
    w, a = pu.on_gpu(tb, p)
    y, xa = tb.tb_packed_linear(w, p["x"].cuda(), a)
    want, xa64, bound = pu.forward64(p)
    pu.near(y, want, bound, what)
    assert pu.norm_off(y, want) <= pu.HALF_STEP[p["dtype"]] + 1e-6
    if a is None:
        assert xa is None
    else:
        pu.near(xa, xa64, (p["d"] + 64) * 2.0 ** -23 * (p["x"].double().abs().amax(1, keepdim=True) * p["d"]), what)
        assert pu.norm_off(xa, xa64) <= 2e-6
        assert not xa[(pu.owners(p) < 0).cuda()].any()
    assert tb.tb_device_error_flag() == 0
    return y, xa


@pytest.mark.parametrize("bits", range(2, 9))
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_tok", [1, 5, 19, 130])
def test_every_width_of_code(bits, dtype, n_tok):
    _forward(pu.problem(bits, n_tok, 152, 384, bits, 128, dtype))


@pytest.mark.parametrize("rows,d,group", [(8, 32, 0), (24, 32, 32), (136, 96, 96), (264, 160, 32), (128, 544, 0), (1032, 128, 64),
                                          (256, 1024, 256), (520, 1152, 384), (16, 2080, 416), (2056, 640, 128)])
@pytest.mark.parametrize("n_tok", [1, 2, 8, 9, 16, 17, 33, 64, 65, 129, 256, 257])
def test_shapes(rows, d, group, n_tok):
    _forward(pu.problem(rows + d, n_tok, rows, d, 3 if rows % 16 else 4, group, BF), (rows, d, group, n_tok))


@pytest.mark.parametrize("rows,d,group", [(24, 32, 0), (264, 160, 32), (520, 1152, 384)])
@pytest.mark.parametrize("n_tok", [1, 9, 70, 300])
def test_shapes_float(rows, d, group, n_tok):
    _forward(pu.problem(rows + d, n_tok, rows, d, 2, group, F32), (rows, d, group, n_tok))


@pytest.mark.parametrize("rows,d,group,bits", [(8, 32, 0, 4), (24, 32, 32, 3), (136, 96, 96, 5), (264, 160, 32, 2), (128, 544, 0, 6), (1032, 128, 64, 4),
                                               (256, 1024, 256, 7), (520, 1152, 384, 8), (16, 2080, 416, 3), (2056, 640, 128, 2)])
@pytest.mark.parametrize("more", [1, 31, 200])
def test_shapes_in_tiles(rows, d, group, bits, more):
    """As many tokens as go to the tensor-core tiles: more than 2^18 results."""
    n_tok = (1 << 18) // rows + more
    _forward(pu.problem(rows + d, n_tok, rows, d, bits, group, BF), (rows, d, group, n_tok))


REQUESTS = {
    "one": (40, [0, 40], [0]),
    "single tokens": (11, list(range(12)), [3, 1, 1, -1, 0, 2, 3, 9, 0, 0, 1]),
    "empty ones": (37, [0, 0, 5, 5, 5, 30, 37, 37], [1, 0, 2, 3, 2, 1, 0]),
    "none": (20, [0, 10, 20], [-1, 4]),
    "gaps at both ends": (50, [7, 9, 31], [2, 0]),
    "ragged": (301, [0, 1, 18, 19, 140, 290, 301], [3, 0, 1, 2, 0, 3]),
    "long": (600, [0, 250, 600], [1, 1]),
}


def _with_adapters(name, rank, dtype, rows=264, d=416, bits=4, group=32):
    n_tok, starts, ids = REQUESTS[name]
    return pu.problem(len(name) + rank, n_tok, rows, d, bits, group, dtype, 4, rank, starts, ids)


@pytest.mark.parametrize("name", REQUESTS)
@pytest.mark.parametrize("rank", [8, 16, 40, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_adapters(name, rank, dtype):
    _forward(_with_adapters(name, rank, dtype), name)


@pytest.mark.parametrize("n_tok,rows,d,n_req,rank", [(64, 2056, 512, 32, 64), (70, 2056, 256, 70, 16), (1100, 264, 416, 3, 8), (1100, 264, 416, 1100, 8),
                                                   (300, 1032, 256, 5, 128), (300, 1032, 1024, 300, 128), (2100, 136, 96, 9, 32)])
def test_adapters_in_tiles(n_tok, rows, d, n_req, rank):
    """Requests in the tiles' own stages and joined to their sums, many and few of them."""
    g = torch.Generator().manual_seed(n_tok + rows)
    cuts = torch.sort(torch.randint(0, n_tok + 1, (n_req - 1,), generator=g)).values.tolist()
    starts = list(range(n_tok + 1)) if n_req == n_tok else [0, *cuts, n_tok]
    _forward(pu.problem(7, n_tok, rows, d, 4, 32, BF, 5, rank, starts, torch.randint(-1, 5, (n_req,), generator=g).tolist()))


@pytest.mark.parametrize("name", REQUESTS)
@pytest.mark.parametrize("rank,dtype", [(8, BF), (40, BF), (128, BF), (16, F32)])
@pytest.mark.parametrize("kept", ["full", "8 bits"])
def test_gradients(name, rank, dtype, kept):
    tb = _tb()
    p = _with_adapters(name, rank, dtype)
    w, a = pu.on_gpu(tb, p)
    xa = pu.forward64(p)[1].float()
    if kept == "full":
        x, how = None, dict(x=p["x"].cuda())
    else:
        codes, scales = pu.eight_bits(p["x"])
        x = torch.from_numpy(codes).double() * torch.from_numpy(scales).double().repeat_interleave(128, 1)[:, :p["d"]]
        how = dict(checkpoint=(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()))
    out = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, xa=xa.cuda(), **how)
    for name_, got in zip(("dx", "dA", "dB"), out):
        want, bound = pu.backward64(p, x, xa)[name_]
        pu.near(got, want, bound, (name, name_))
        if name_ != "dx" and want.any():
            assert pu.norm_off(got, want) <= 3e-6, name_
    again = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, xa=xa.cuda(), **how)
    assert all(torch.equal(g, h) for g, h in zip(out, again))
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("rows,d,group,bits", [(8, 32, 0, 2), (136, 96, 96, 3), (264, 160, 32, 5), (1032, 544, 0, 7), (256, 1024, 128, 8),
                                               (520, 1152, 384, 6)])
@pytest.mark.parametrize("n_tok", [1, 16, 33, 129, 260])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_input_gradient_alone(rows, d, group, bits, n_tok, dtype):
    tb = _tb()
    p = pu.problem(rows, n_tok, rows, d, bits, group, dtype)
    w, _ = pu.on_gpu(tb, p)
    dx, dA, dB = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    assert dA is None and dB is None
    want, bound = pu.backward64(p)["dx"]
    pu.near(dx, want, bound)
    assert pu.norm_off(dx, want) <= (1.5 * pu.HALF_STEP[dtype] if dtype == BF else 2e-6)


def test_gradients_against_differences():
    """dx, dA and dB are the slopes of sum(y * g): the function is linear in x and in each adapter matrix, so a difference of any
    step is exact up to rounding (float, steps of the values' own size)."""
    tb = _tb()
    p = pu.problem(3, 29, 40, 64, 4, 32, F32, 2, 8, [0, 11, 29], [1, 0])
    g = p["dy"].double()

    def value(q):
        w, a = pu.on_gpu(tb, q)
        return (tb.tb_packed_linear(w, q["x"].cuda(), a)[0].cpu().double() * g).sum()

    w, a = pu.on_gpu(tb, p)
    y, xa = tb.tb_packed_linear(w, p["x"].cuda(), a)
    grads = dict(zip(("x", "A", "B"), tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, x=p["x"].cuda(), xa=xa)))
    r = torch.Generator().manual_seed(5)
    for name, grad in grads.items():
        step = torch.randn(p[name].shape, generator=r)
        up, down = dict(p), dict(p)
        up[name], down[name] = p[name] + step, p[name] - step
        slope = (value(up) - value(down)) / 2
        want = (grad.cpu().double() * step.double()).sum()
        # 29 x 40 outputs of sums of 64 + 8 products, a few units in magnitude, each in float
        assert abs(slope - want) <= 1e-5 * (g.abs().sum() + abs(want)), name


def test_a_run_of_them_as_in_training():
    """Forward, the input kept in 8 bits, backward from it: the adapters' gradients are those of the decoded input."""
    tb = _tb()
    n_tok, starts, ids = REQUESTS["ragged"]
    p = pu.problem(9, n_tok, 392, 640, 2, 128, BF, 4, 16, starts, ids)
    w, a = pu.on_gpu(tb, p)
    x = p["x"].cuda()
    y, xa = tb.tb_packed_linear(w, x, a)
    kept = tb.tb_checkpoint_pack(x)
    del x
    dx, dA, dB = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, checkpoint=kept, xa=xa)
    x8 = tb.tb_checkpoint_unpack(*kept, dtype=F32).cpu()
    assert (x8.double() - p["x"].double()).abs().max() <= 0.5 * kept[1].max().item() * 1.0001
    want = pu.backward64(p, x8, xa.cpu())
    for name, got in (("dx", dx), ("dA", dA), ("dB", dB)):
        pu.near(got, *want[name], name)
    yw, _, bound = pu.forward64(p)
    pu.near(y, yw, bound)


def test_quantized_layer_to_product():
    """From the quantizer's own outputs: codes packed, the product is that with the dequantized weights."""
    import numpy as np
    import parity_util as qu
    tb = _tb()
    prob = qu.make_problem(1, 256, 2, 32, 1024, with_r=False)
    res = qu.run_gpu(prob, 3, 128, 8, 3)
    t = lambda v: torch.from_numpy(np.ascontiguousarray(v))  # noqa: E731
    packed = tb.tb_pack_codes(t(res["codes"]).cuda(), 3)
    w = tb.packed_weight(packed, t(res["scales"]).cuda(), t(res["zeros"]).cuda(), 256, 3, 128)
    x = torch.randn((21, 256), generator=torch.Generator().manual_seed(2)).to(BF)
    y, _ = tb.tb_packed_linear(w, x.cuda())
    Q = t(res["scales"]).double().repeat_interleave(128, 1) * (t(res["codes"]).double() - t(res["zeros"]).double().repeat_interleave(128, 1))
    want = x.double() @ Q.T
    pu.near(y, want, pu.HALF_STEP[BF] * want.abs() + pu.sum_bound(256, x.double().abs() @ Q.abs().T, BF))


@pytest.mark.parametrize("n_tok,starts", [(24, [0, 3, 9, 24]), (200, [0, 50, 133, 200])])
@pytest.mark.parametrize("rank", [8, 64])
def test_what_is_not_finite_stays_with_its_own(n_tok, starts, rank):
    """An infinite or undefined activation changes its own token alone, and one in an adapter its requests alone."""
    tb = _tb()
    ids = [1, 0, 1]
    p = pu.problem(4, n_tok, 264, 256, 4, 128, BF, 3, rank, starts, ids)
    p["x"][starts[1] + 2, 17] = float("inf")
    p["x"][starts[1] + 4, 200] = float("nan")
    p["A"][2] = float("nan")                       # no request has this one
    clean = dict(p, A=p["A"].clone(), B=p["B"].clone(), x=p["x"].clone())
    clean["x"][starts[1] + 2, 17], clean["x"][starts[1] + 4, 200] = 0.0, 0.0
    p["B"][0, 3, 100] = float("inf")
    w, a = pu.on_gpu(tb, p)
    y, xa = (v.cpu() for v in tb.tb_packed_linear(w, p["x"].cuda(), a))
    want, xa64, bound = pu.forward64(clean)
    hit = torch.zeros(n_tok, dtype=torch.bool)
    hit[[starts[1] + 2, starts[1] + 4]] = True
    own0 = pu.owners(p) == 0
    fine = ~hit
    assert ((y[fine].double() - want[fine]).abs() <= bound[fine])[:, :100].all()
    assert ((y[fine].double() - want[fine]).abs() <= bound[fine])[:, 101:].all()
    assert torch.isfinite(y[fine & ~own0]).all() and not torch.isfinite(y[own0][:, 100]).any()
    # 0 is among the values of c - z, so an infinite activation gives what is no number or an infinity in every column
    assert not torch.isfinite(y[hit]).any() and not torch.isfinite(xa[hit]).any() and torch.isfinite(xa[fine]).all()
    # backward: an undefined token of one adapter leaves the other adapters' gradients alone
    q = dict(clean, dy=p["dy"].clone())
    q["dy"][starts[1] + 2, 5] = float("nan")
    w, a = pu.on_gpu(tb, q)
    x = q["x"].clone()
    x[starts[1] + 3, 9] = float("inf")
    dx, dA, dB = tb.tb_packed_linear_backward(w, q["dy"].cuda(), a, x=x.cuda(), xa=xa64.float().cuda())
    ref = pu.backward64(q, None, xa64.float())
    for got, name in ((dA, "dA"), (dB, "dB")):
        pu.near(got[1], ref[name][0][1], ref[name][1][1], name)
        assert not got[2].any()
        assert torch.isnan(got[0]).any()
    rows = torch.ones(n_tok, dtype=torch.bool)
    rows[starts[1] + 2] = False
    pu.near(dx[rows.cuda()], ref["dx"][0][rows], ref["dx"][1][rows], "dx")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_tokens(dtype):
    tb = _tb()
    p = pu.problem(1, 0, 64, 96, 3, 32, dtype, 2, 8, [0, 0], [1])
    w, a = pu.on_gpu(tb, p)
    y, xa = tb.tb_packed_linear(w, p["x"].cuda(), a)
    assert y.shape == (0, 64) and xa.shape == (0, 8)
    dx, dA, dB = tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, x=p["x"].cuda(), xa=xa)
    assert dx.shape == (0, 96) and not dA.any() and not dB.any()
    codes, scales = tb.tb_checkpoint_pack(p["x"].cuda())
    assert tb.tb_checkpoint_unpack(codes, scales).shape == (0, 96)


@pytest.mark.parametrize("n_tok", [3, 40, 333])
def test_captured_and_on_another_stream(n_tok):
    """Two captured graphs and eager calls between their replays: each sees its own inputs, bits as from an eager call."""
    tb = _tb()
    starts, ids = [0, n_tok // 2, n_tok], [1, 0]
    probs = [pu.problem(s, n_tok, 264, 512, 2, 128, BF, 2, 16, starts, ids) for s in (1, 2)]
    want, graphs, outs, ins = [], [], [], []
    for p in probs:
        w, a = pu.on_gpu(tb, p)
        x, dy = p["x"].cuda(), p["dy"].cuda()

        def call(w=w, a=a, x=x, dy=dy):
            y, xa = tb.tb_packed_linear(w, x, a)
            kept = tb.tb_checkpoint_pack(x)
            return (y, xa) + tb.tb_packed_linear_backward(w, dy, a, checkpoint=kept, xa=xa)

        want.append(call())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = call()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(u, v) for u, v in zip(other, want[-1]))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
        ins.append((x, dy, w, a))   # a graph holds addresses: what it reads has to live on
    for k in (0, 1, 1, 0):
        for t in outs[k]:
            t.zero_()
        graphs[k].replay()
        tb.tb_packed_linear(w, x, a)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(outs[k], want[k]))
    ins[0][0].copy_(ins[1][0])                      # new inputs in the captured buffers
    graphs[0].replay()
    torch.cuda.synchronize()
    w, a = pu.on_gpu(tb, probs[0])
    assert torch.equal(outs[0][0], tb.tb_packed_linear(w, ins[1][0], a)[0])


def test_neighbours_of_the_outputs_stay():
    """Guard values before and behind every output."""
    tb = _tb()
    for n_tok in (3, 21, 150):
        p = pu.problem(n_tok, n_tok, 136, 160, 3, 32, BF, 1, 8, [0, n_tok], [0])
        w, a = pu.on_gpu(tb, p)
        buf = torch.full((n_tok * 136 + 128,), 7.0, dtype=BF, device="cuda")
        low = torch.full((n_tok * 8 + 128,), 7.0, device="cuda")
        y, xa = buf[64:64 + n_tok * 136].view(n_tok, 136), low[64:64 + n_tok * 8].view(n_tok, 8)
        tb.tb_packed_linear(w, p["x"].cuda(), a, y=y, xa=xa)
        want, xa64, bound = pu.forward64(p)
        pu.near(y, want, bound)
        for b, n in ((buf, n_tok * 136), (low, n_tok * 8)):
            assert (b[:64] == 7).all() and (b[64 + n:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_tok,d", [(1, 32), (3, 96), (5, 128), (17, 160), (33, 4096), (257, 1184)])
def test_8_bit_form(n_tok, d, dtype):
    tb = _tb()
    x = pu.problem(n_tok, n_tok, 8, d, 2, 0, dtype)["x"]
    if n_tok > 2:
        x[1] = 0.0
        x[2] *= 1e-38
        x[0, :min(d, 128)] = torch.arange(min(d, 128)) * 0.5      # ties: the quotients are halves where the scale is 1
        x[0, 0] = 127.0
    codes, scales = tb.tb_checkpoint_pack(x.cuda())
    cw, sw = pu.eight_bits(x)
    assert (scales.cpu().numpy() == sw).all() and (codes.cpu().numpy() == cw).all()
    got = tb.tb_checkpoint_unpack(codes, scales, dtype)
    want = (torch.from_numpy(cw).float() * torch.from_numpy(sw).repeat_interleave(128, 1)[:, :d]).to(dtype)
    assert torch.equal(got.cpu(), want)


def test_8_bit_form_of_what_is_not_finite():
    tb = _tb()
    x = torch.ones((4, 288), dtype=BF)
    x[0, 130], x[1, 0], x[2, 287] = float("inf"), float("nan"), float("-inf")
    codes, scales = tb.tb_checkpoint_pack(x.cuda())
    v = tb.tb_checkpoint_unpack(codes, scales, F32).cpu()
    bad = torch.zeros((4, 3), dtype=torch.bool)
    bad[0, 1] = bad[1, 0] = bad[2, 2] = True
    assert torch.equal(torch.isnan(scales).cpu(), bad)
    assert torch.equal(torch.isnan(v), bad.repeat_interleave(128, 1)[:, :288])
    assert ((v[3] - 1).abs() < 1e-6).all()


@pytest.mark.parametrize("n_tok,rows,d,rank,n_req,seed", [(24, 136, 640, 16, 24, 0), (32, 1032, 1024, 24, 9, 1), (40, 264, 2048, 16, 40, 2),
                                                          (64, 520, 4096, 8, 64, 3), (100, 264, 3584, 64, 7, 4), (257, 1544, 1024, 16, 60, 5),
                                                          (700, 264, 384, 8, 600, 6), (640, 2056, 256, 40, 5, 7)])
def test_many_requests(n_tok, rows, d, rank, n_req, seed):
    """Requests of every length at the sizes where tiles, splits of the contraction and the adapters' ways change."""
    tb = _tb()
    r = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(0, n_tok + 1, (n_req - 1,), generator=r))[0].tolist()
    starts = list(range(n_tok + 1)) if n_req == n_tok else [0] + cuts + [n_tok]
    ids = torch.randint(-1, 12, (n_req,), generator=r).tolist()
    p = pu.problem(seed, n_tok, rows, d, 2 + seed % 4, 128, BF, 11, rank, starts, ids)
    _forward(p)
    w, a = pu.on_gpu(tb, p)
    xa = pu.forward64(p)[1].float()
    want = pu.backward64(p, None, xa)
    for got, name in zip(tb.tb_packed_linear_backward(w, p["dy"].cuda(), a, x=p["x"].cuda(), xa=xa.cuda()), ("dx", "dA", "dB")):
        pu.near(got, *want[name], name)
    assert tb.tb_device_error_flag() == 0


def test_more_adapters_in_a_tile_than_fit_side_by_side():
    starts = [0, 10, 20, 30, 40, 50, 60, 70, 80, 600]
    _forward(pu.problem(8, 600, 136, 4096, 4, 128, BF, 9, 128, starts, [3, 1, 4, 8, 5, 0, 2, 6, 7]))


@pytest.mark.parametrize("rank", [8, 128])
def test_long_contractions_of_the_narrow_product(rank):
    """A CTA with 8192 columns ends its accumulations on the way; the reference in double on the GPU."""
    tb = _tb()
    n_tok, d = 10100, 8192
    p = pu.problem(5, 1, 8, d, 2, 0, BF, 2, rank, [0, 1], [0])
    w, _ = pu.on_gpu(tb, p)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n_tok, d), generator=g, device="cuda").to(BF)
    starts, ids = torch.tensor([0, 4000, n_tok], dtype=torch.int32).cuda(), torch.tensor([1, 0], dtype=torch.int32).cuda()
    A, B = p["A"].cuda(), p["B"].cuda()
    y, xa = tb.tb_packed_linear(w, x, tb.adapters(A, B, p["scale"].cuda(), starts, ids))
    want = torch.cat([x[:4000].double() @ A[1].double().T, x[4000:].double() @ A[0].double().T])
    # a step of 16 columns may drop up to 2^-23 of the running sum, which averages 2/3 of the final one (it grows like a root); an
    # accumulation has 32 steps, or with ranks above 32 as many as a quarter of the 8192 columns has: 128
    assert ((xa - want).norm() / want.norm()).item() <= 2 / 3 * (32 if rank == 8 else 128) * 2.0 ** -23
    assert (xa - want).abs().max().item() <= (d + 64) * 2.0 ** -23 * (x.double().abs() @ A.double().abs().amax(0).T).max().item()
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("rank", [16, 64, 128])
@pytest.mark.parametrize("kept", ["full", "8 bits"])
def test_gradients_of_many_tokens(rank, kept):
    """A CTA with more than 2048 tokens ends its accumulations on the way; the reference in double on the GPU."""
    tb = _tb()
    n_tok, d, rows = 21003, 128, 136
    p = pu.problem(6, 1, rows, d, 4, 0, BF, 2, rank, [0, 1], [0])
    w, _ = pu.on_gpu(tb, p)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn((n_tok, n), generator=g, device="cuda").to(BF) for n in (d, rows))
    xa = torch.randn((n_tok, rank), generator=g, device="cuda")
    starts, ids = torch.tensor([0, 20000, n_tok], dtype=torch.int32).cuda(), torch.tensor([1, 0], dtype=torch.int32).cuda()
    A, B, c = p["A"].cuda(), p["B"].cuda(), p["scale"].cuda()
    codes = tb.tb_checkpoint_pack(x)
    how = dict(x=x) if kept == "full" else dict(checkpoint=codes)
    xin = x.double() if kept == "full" else codes[0].double() * codes[1].double()
    _, dA, dB = tb.tb_packed_linear_backward(w, dy, tb.adapters(A, B, c, starts, ids), xa=xa, want_dx=False, **how)
    for i, tok in ((1, slice(0, 20000)), (0, slice(20000, n_tok))):
        u = c[i].double() * (dy[tok].double() @ B[i].double().T)
        for got, want in ((dA[i], u.T @ xin[tok]), (dB[i], c[i].double() * (xa[tok].double().T @ dy[tok].double()))):
            assert ((got - want).norm() / want.norm()).item() <= 3e-6
    assert tb.tb_device_error_flag() == 0


def test_offsets_beyond_32_bits():
    """270 000 tokens of 8192 columns: 2.2e9 values.  The first, a middle and the last tokens against a call on them alone."""
    tb = _tb()
    n_tok, d, rows = 270000, 8192, 8
    p = pu.problem(7, 1, rows, d, 2, 128, BF, 1, 8, [0, 1], [0])
    w, _ = pu.on_gpu(tb, p)
    x = torch.empty((n_tok, d), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    for t in range(0, n_tok, 30000):
        x[t:t + 30000].normal_(generator=g)
    dy = torch.randn((n_tok, rows), generator=g, device="cuda").to(BF)
    def batch(n):
        return tb.adapters(p["A"].cuda(), p["B"].cuda(), p["scale"].cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(),
                           torch.tensor([0], dtype=torch.int32).cuda())
    y, xa = tb.tb_packed_linear(w, x, batch(n_tok))
    dx, _, _ = tb.tb_packed_linear_backward(w, dy, batch(n_tok))
    codes, scales = tb.tb_checkpoint_pack(x)
    for t in (0, 131072, n_tok - 64):
        s = slice(t, t + 64)
        y1, xa1 = tb.tb_packed_linear(w, x[s].clone(), batch(64))
        assert (y[s].float() - y1.float()).norm() <= 0.01 * y1.float().norm() and (xa[s] - xa1).norm() <= 1e-5 * xa1.norm()
        dx1, _, _ = tb.tb_packed_linear_backward(w, dy[s].clone(), batch(64))
        assert (dx[s].float() - dx1.float()).norm() <= 0.01 * dx1.float().norm()
        c1, s1 = tb.tb_checkpoint_pack(x[s].clone())
        assert torch.equal(codes[s], c1) and torch.equal(scales[s], s1)
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("bits,n_tok", [(2, 5), (3, 70), (4, 70), (7, 5), (7, 70), (8, 5), (8, 70)])
def test_zero_points_outside_the_codes(bits, n_tok):
    p = pu.problem(bits, n_tok, 136, 256, bits, 128, BF)
    z = torch.randint(-128, 129, p["zeros"].shape, generator=torch.Generator().manual_seed(bits), dtype=torch.int32)
    zd = (p["zeros"] - z).double().repeat_interleave(128, 1) * p["scales"].double().repeat_interleave(128, 1)
    p["zeros"], p["Q"] = z, p["Q"] + zd
    if bits < 8:
        _forward(p)
        return
    # codes up to 255: c - z goes beyond 256 and is rounded to bf16, by 2^-8 of it at most, which is 2^-8 of the product's magnitudes
    tb = _tb()
    w, _ = pu.on_gpu(tb, p)
    want, _, bound = pu.forward64(p)
    pu.near(tb.tb_packed_linear(w, p["x"].cuda())[0], want, bound + 1.01 * 2.0 ** -8 * (p["x"].double().abs() @ p["Q"].abs().T))


def test_refusals():
    tb = _tb()
    p = pu.problem(1, 40, 64, 128, 4, 0, BF, 2, 8, [0, 40], [0])
    w, a = pu.on_gpu(tb, p)
    x, dy = p["x"].cuda(), p["dy"].cuda()
    xa = torch.zeros((40, 8), device="cuda")
    bad = [lambda: tb.tb_packed_linear(w, p["x"], a), lambda: tb.tb_packed_linear(w, x.half(), a), lambda: tb.tb_packed_linear(w, x.float(), a),
           lambda: tb.tb_packed_linear(w, x[:, :96].contiguous()), lambda: tb.tb_packed_linear(w, x.T.contiguous().T),
           lambda: tb.tb_packed_linear(w, x, y=dy[:3]), lambda: tb.tb_packed_linear(w, x, a, xa=xa[:, :4]),
           lambda: tb.tb_packed_linear(w, x, y=dy.float()), lambda: tb.tb_packed_linear_backward(w, x),
           lambda: tb.tb_packed_linear_backward(w, dy, a, x=x), lambda: tb.tb_packed_linear_backward(w, dy, a, x=x[:20], xa=xa),
           lambda: tb.tb_packed_linear_backward(w, dy, a, x=x.float(), xa=xa), lambda: tb.tb_checkpoint_pack(p["x"]),
           lambda: tb.tb_checkpoint_pack(x.half()), lambda: tb.tb_checkpoint_unpack(x.to(torch.int8), xa),
           lambda: tb.tb_packed_linear(w, x, ws=torch.empty(1 << 20, dtype=torch.uint8))]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    both = tb.tb_checkpoint_pack(x)
    for call, status in ((lambda: tb.tb_packed_linear_backward(w, dy, a, x=x, xa=xa, ws=torch.empty(256, dtype=torch.uint8, device="cuda")), 3),
                         (lambda: tb.tb_packed_linear_backward(w, dy, a, x=x, checkpoint=both, xa=xa), 1),
                         (lambda: tb.tb_packed_linear_backward(w, dy, want_dx=False), 1)):
        with pytest.raises(tb.TurboBoAError) as e:
            call()
        assert e.value.status == status
    need = tb.load().tb_packed_linear_workspace(w.address, a.address, 1, 40)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    y, _ = tb.tb_packed_linear(w, x, a, ws=ws)
    assert torch.equal(y, tb.tb_packed_linear(w, x, a)[0])
    need = tb.load().tb_packed_linear_backward_workspace(w.address, a.address, 1, 40)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    got = tb.tb_packed_linear_backward(w, dy, a, x=x, xa=xa, ws=ws)
    assert all(torch.equal(u, v) for u, v in zip(got, tb.tb_packed_linear_backward(w, dy, a, x=x, xa=xa)))


@pytest.mark.parametrize("n_tok,rows,d,bits,group", [(20000, 40, 520 - 8, 2, 0), (9000, 264, 96, 3, 96), (33000, 8, 160, 7, 32), (5000, 1032, 1056, 4, 0)])
def test_many_tiles_for_every_pair_of_processors(n_tok, rows, d, bits, group):
    """Short contractions and many tiles, with adapters' stages between them; the reference in double on the GPU."""
    tb = _tb()
    rank = 24
    p = pu.problem(11, 1, rows, d, bits, group, BF, 3, rank, [0, 1], [0])
    w, _ = pu.on_gpu(tb, p)
    g = torch.Generator(device="cuda").manual_seed(12)
    x, dy = (torch.randn((n_tok, n), generator=g, device="cuda").to(BF) for n in (d, rows))
    cuts = torch.sort(torch.randint(0, n_tok, (149,), generator=g, device="cuda"))[0].tolist()
    ids = torch.randint(-1, 3, (150,), generator=g, device="cuda")
    at = [0] + cuts + [n_tok]
    a = tb.adapters(p["A"].cuda(), p["B"].cuda(), p["scale"].cuda(), torch.tensor(at, dtype=torch.int32).cuda(), ids.to(torch.int32))
    Q, A, B, c = p["Q"].cuda(), p["A"].cuda().double(), p["B"].cuda().double(), p["scale"].cuda().double()
    y64, dx64 = x.double() @ Q.T, dy.double() @ Q
    for j, i in enumerate(ids.tolist()):
        if i >= 0:
            s = slice(at[j], at[j + 1])
            y64[s] += c[i] * ((x[s].double() @ A[i].T) @ B[i])
            dx64[s] += c[i] * ((dy[s].double() @ B[i].T) @ A[i])
    for _ in range(3):
        y, xa = tb.tb_packed_linear(w, x, a)
        dx, dA, dB = tb.tb_packed_linear_backward(w, dy, a, x=x, xa=xa)
        assert tb.tb_device_error_flag() == 0
        # every token by itself: a rounding of its values, backward one of the weights too
        assert ((y - y64).norm(dim=1) <= 1.01 * 2.0 ** -8 * y64.norm(dim=1) + 1e-30).all()
        assert ((dx - dx64).norm(dim=1) <= 2.02 * 2.0 ** -8 * dx64.norm(dim=1) + 2.0 ** -8 * dy.double().norm(dim=1) * Q.norm(dim=1).max()).all()


@pytest.mark.parametrize("group", [32, 128, 0])
@pytest.mark.parametrize("n_tok", [3, 40, 97, 200])
def test_what_is_not_finite_in_float(n_tok, group):
    """Infinite and undefined activations stay with their token and become what the formula says; the largest floats stay finite."""
    tb = _tb()
    p = pu.problem(4, n_tok, 264, 256, 4, group, F32)
    clean = p["x"].clone(), p["dy"].clone()
    hit = torch.zeros(n_tok, dtype=torch.bool)
    hit[:2] = True
    p["x"][0, 17], p["x"][1, 200] = float("inf"), float("nan")
    p["dy"][0, 30], p["dy"][1, 263] = float("-inf"), float("nan")
    w, _ = pu.on_gpu(tb, p)
    y, _ = tb.tb_packed_linear(w, p["x"].cuda())
    dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    q = dict(p, x=clean[0], dy=clean[1])
    want, _, bound = pu.forward64(q)
    pu.near(y.cpu()[~hit], want[~hit], bound[~hit], "y")
    ref = pu.backward64(q, None, None)["dx"]
    pu.near(dx.cpu()[~hit], ref[0][~hit], ref[1][~hit], "dx")
    Q = p["Q"]
    for got, v, k in ((y, p["x"], Q.T), (dx, p["dy"], Q)):
        got = got.cpu()
        assert torch.isnan(got[1]).all()
        at = int(torch.isinf(v[0]).nonzero()[0])
        zero = k[at] == 0
        assert torch.isnan(got[0][zero]).all()
        assert torch.equal(got[0][~zero].double(), (v[0, at].double() * k[at])[~zero])


@pytest.mark.parametrize("bits,group", [(4, 128), (4, 32), (7, 0)])
@pytest.mark.parametrize("n_tok", [5, 130])
def test_zero_points_outside_the_codes_in_float(bits, group, n_tok):
    p = pu.problem(bits, n_tok, 136, 256, bits, group, F32)
    z = torch.randint(-128, 129, p["zeros"].shape, generator=torch.Generator().manual_seed(bits), dtype=torch.int32)
    wide = lambda v: v.double().repeat_interleave(p["d"] // v.shape[1], 1)  # noqa: E731
    p["Q"] = p["Q"] + wide(p["zeros"] - z) * wide(p["scales"])
    p["zeros"] = z
    _forward(p)
    tb = _tb()
    w, _ = pu.on_gpu(tb, p)
    dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    ref = pu.backward64(p, None, None)["dx"]
    pu.near(dx, ref[0], ref[1], "dx")


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n_tok", [20, 100])
def test_long_contractions_in_float(n_tok, group):
    """Sums of 32 columns, in six (24 for few tokens: sums of 128) steps of the matrix unit that drop less than 2^-23 of a sum each, and 256
    (64) float additions, each off by 2^-24 at most: in the mean of all values at most (2 * 24 + 8) 2^-24 or (2 * 6 + 16) 2^-24, since
    the errors of different sums have nothing to do with one another.  (A warp's own sums in the kernel for few tokens are shorter.)"""
    tb = _tb()
    p = pu.problem(n_tok, n_tok, 8192, 8192, 4, group, F32)
    w, _ = pu.on_gpu(tb, p)
    y, _ = tb.tb_packed_linear(w, p["x"].cuda())
    dx, _, _ = tb.tb_packed_linear_backward(w, p["dy"].cuda())
    Q = p["Q"].cuda()
    tol = {True: 2 * 24 + 8, False: 2 * 6 + 16}
    for got, v, k, few in ((y, p["x"], Q.T, n_tok <= 96), (dx, p["dy"], Q, False)):
        want = v.cuda().double() @ k
        assert float((got.double() - want).norm() / want.norm()) <= tol[few] * 2.0 ** -24


@pytest.mark.parametrize("n_tok,d,n_req,rank", [(22000, 96, 5, 128), (9000, 416, 150, 80), (3001, 1184, 60, 128), (17000, 2080, 3, 8), (2100, 1056, 1, 128)])
def test_narrow_product_in_tiles(n_tok, d, n_req, rank):
    g = torch.Generator().manual_seed(n_tok)
    starts = [3, *torch.sort(torch.randint(3, n_tok - 5, (n_req - 1,), generator=g)).values.tolist(), n_tok - 5]
    ids = torch.randint(-1, 7, (n_req,), generator=g).tolist()
    ids[-1] = 2
    _forward(pu.problem(7, n_tok, 40, d, 4, 32, BF, 7, rank, starts, ids))


@pytest.mark.parametrize("n_tok,rows,d,rank,dtype", [(24, 264, 512, 16, BF), (70, 4104, 1024, 64, BF), (400, 1032, 768, 32, BF), (2300, 264, 1056, 128, BF), (130, 264, 512, 16, F32)])
def test_calls_one_after_the_other_and_side_by_side(n_tok, rows, d, rank, dtype):
    """Calls that take the same outputs and scratch in turn, and calls of two streams at once, give the bits of a call by itself."""
    tb = _tb()
    n_req = 5
    cuts = torch.sort(torch.randint(0, n_tok + 1, (n_req - 1,), generator=torch.Generator().manual_seed(n_tok))).values.tolist()
    p = pu.problem(n_tok, n_tok, rows, d, 4, 32, dtype, 3, rank, [0, *cuts, n_tok], [0, 2, 1, 0, 2])
    w, a = pu.on_gpu(tb, p)
    xs = [p["x"].cuda() * s for s in (1.0, -2.0, 0.5, 4.0)]
    dys = [p["dy"].cuda() * s for s in (1.0, 0.5, -2.0, 1.0)]

    def one(x, dy, **kept):
        y, xa = tb.tb_packed_linear(w, x, a, **kept)
        dx, dA, dB = tb.tb_packed_linear_backward(w, dy, a, x=x, xa=xa, ws=kept.get("ws"))
        return [v.clone() for v in (y, xa, dx, dA, dB)]

    alone = []
    for x, dy in zip(xs, dys):
        alone.append(one(x, dy))
        torch.cuda.synchronize()
    lib, t = tb.load(), {BF: 1, F32: 0}[dtype]
    need = max(lib.tb_packed_linear_workspace(w.address, a.address, t, n_tok), lib.tb_packed_linear_backward_workspace(w.address, a.address, t, n_tok))
    kept = dict(ws=torch.empty(need, dtype=torch.uint8, device="cuda"), y=torch.empty_like(alone[0][0]), xa=torch.empty_like(alone[0][1]))
    for _ in range(5):
        got = [one(x, dy, **kept) for x, dy in zip(xs, dys)]
        assert all(torch.equal(u, v) for g, s in zip(got, alone) for u, v in zip(g, s))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for k in range(12):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(one(xs[(k + i) % 4], dys[(k + i) % 4]))
    torch.cuda.synchronize()
    for i in range(2):
        for k in range(12):
            assert all(torch.equal(u, v) for u, v in zip(got[i][k], alone[(k + i) % 4])), (i, k)
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("n_tok,rows,d,bits,group,rank", [(208, 832, 2688, 4, 128, 128), (40, 136, 384, 4, 128, 8), (300, 1160, 128, 3, 0, 16), (70, 264, 640, 8, 128, 8),
                                                        (1100, 264, 384, 2, 384, 8), (90, 200, 96, 5, 96, 16), (24, 136, 1152, 7, 128, 16), (1, 8, 32, 2, 32, 8)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_inputs_and_scratch_that_end_with_their_memory(n_tok, rows, d, bits, group, rank, dtype):
    """Every array at the very end of an allocation of its own: nothing behind it is read (columns of a tile behind the matrix, for
    instance, whose zero-points no group has)."""
    tb = _tb()
    hold = []

    def at_the_end(v):
        n = v.numel() * v.element_size()
        room = torch.empty(max(16 << 20, (n + (2 << 20) - 1) >> 21 << 21), dtype=torch.uint8, device="cuda")
        hold.append(room)
        to = room[(room.numel() - n) // 256 * 256:][:n].view(v.dtype).view(v.shape)
        to.copy_(v)
        return to

    p = pu.problem(n_tok + rows, n_tok, rows, d, bits, group, dtype, 2, rank, sorted([0, n_tok // 3, n_tok // 2, n_tok]), [1, 0, 1])
    w0, a0 = pu.on_gpu(tb, p)
    w = tb.packed_weight(*(at_the_end(v) for v in w0.tensors), d, bits, group)
    a = tb.adapters(*(at_the_end(v) for v in a0.tensors))
    x, dy = at_the_end(p["x"].cuda()), at_the_end(p["dy"].cuda())
    lib, t = tb.load(), {BF: 1, F32: 0}[dtype]

    def scratch(size):
        return at_the_end(torch.zeros(max(256, (size + 255) // 256 * 256), dtype=torch.uint8, device="cuda"))

    y, xa = tb.tb_packed_linear(w, x, a, ws=scratch(lib.tb_packed_linear_workspace(w.address, a.address, t, n_tok)))
    want, xa64, bound = pu.forward64(p)
    pu.near(y, want, bound, "y")
    plain, _ = tb.tb_packed_linear(w, x, None, ws=scratch(lib.tb_packed_linear_workspace(w.address, None, t, n_tok)))
    assert torch.isfinite(plain).all()
    codes, scales = (at_the_end(v) for v in tb.tb_checkpoint_pack(x))
    assert torch.isfinite(tb.tb_checkpoint_unpack(codes, scales, dtype)).all()
    xa = at_the_end(xa)
    ref = pu.backward64(p, None, xa.cpu())
    for kept in (dict(x=x), dict(checkpoint=(codes, scales))):
        dx, dA, dB = tb.tb_packed_linear_backward(w, dy, a, xa=xa, ws=scratch(lib.tb_packed_linear_backward_workspace(w.address, a.address, t, n_tok)), **kept)
        pu.near(dx, ref["dx"][0], ref["dx"][1], "dx")
        pu.near(dB, ref["dB"][0], ref["dB"][1], "dB")
    assert tb.tb_device_error_flag() == 0


@pytest.mark.parametrize("n_tok,rows,d,rank,n_req,dtype", [(70, 4104, 1024, 64, 40, BF), (400, 1032, 768, 32, 3, BF), (2300, 264, 1056, 128, 4, BF), (130, 264, 512, 16, 5, F32)])
def test_tiles_captured_and_between_guards(n_tok, rows, d, rank, n_req, dtype):
    """The paths of many tokens in a graph, replayed with other inputs beside eager calls; outputs in the middle of guard values."""
    tb = _tb()
    cuts = torch.sort(torch.randint(0, n_tok + 1, (n_req - 1,), generator=torch.Generator().manual_seed(n_tok))).values.tolist()
    ids = torch.randint(-1, 3, (n_req,), generator=torch.Generator().manual_seed(rows)).tolist()
    p = pu.problem(n_tok, n_tok, rows, d, 4, 32, dtype, 3, rank, [0, *cuts, n_tok], ids)
    w, a = pu.on_gpu(tb, p)
    x, dy = p["x"].cuda(), p["dy"].cuda()
    buf = torch.full((n_tok * rows + 256,), 7.0, dtype=dtype, device="cuda")
    low = torch.full((n_tok * rank + 256,), 7.0, device="cuda")
    y, xa = buf[128:128 + n_tok * rows].view(n_tok, rows), low[128:128 + n_tok * rank].view(n_tok, rank)

    def call(**to):
        out, kept = tb.tb_packed_linear(w, x, a, **to)
        return (out, kept, *tb.tb_packed_linear_backward(w, dy, a, x=x, xa=kept))

    first = [v.clone() for v in call()]
    call(y=y, xa=xa)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = call(y=y, xa=xa)
    for k in range(4):
        x.mul_(-2.0), dy.mul_(0.5)
        want = [v.clone() for v in call()]
        for v in outs:
            v.zero_()
        g.replay()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(outs, want)), k
    assert not torch.equal(outs[0], first[0])
    for b in (buf, low):
        assert (b[:128] == 7).all() and (b[-128:] == 7).all()
    assert tb.tb_device_error_flag() == 0
