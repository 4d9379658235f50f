"""The product with bias, activation and residual on the way to C.

Where every step behind the sum is one operation of float (bias, ReLU, residual, rounding to 16 bits), C is compared bit for bit with
the same steps behind mmm_matmul, whose parity has its own tests; every kernel, tile and split of K goes through that.  Smooth activations
are compared with the formula in 64 bits.  Bound there: the sum is within 1e-5 of the sum of magnitudes (the stated bound of float sums), an
activation's slope is at most 1.13, and its own value is off by a few roundings: 16 * 2^-24 of 1 + |z| and of the residual."""
import math

import pytest
import torch

import paper_2402_14118_amd as mm

T = {"f32": (mm.MMM_F32, torch.float32), "bf16": (mm.MMM_BF16, torch.bfloat16), "f16": (mm.MMM_F16, torch.float16), "f64": (mm.MMM_F64, torch.float64)}
ACTS = {"none": mm.MMM_ACT_NONE, "relu": mm.MMM_ACT_RELU, "gelu": mm.MMM_ACT_GELU, "gelu_tanh": mm.MMM_ACT_GELU_TANH, "silu": mm.MMM_ACT_SILU}
U = 2.0 ** -24


def words(flags):
    rows, cols = flags.shape
    padded = torch.zeros(rows, (cols + 63) // 64 * 64, dtype=torch.uint8)
    padded[:, :cols] = flags
    by = (padded.view(rows, -1, 8) * torch.tensor([1, 2, 4, 8, 16, 32, 64, 128], dtype=torch.uint8)).sum(-1, dtype=torch.uint8)
    return by.view(torch.int64).contiguous().cuda()


def room(M, N, dtype, pad=0, start=0):
    """M x N elements whose rows are `pad` apart and that begin `start` elements behind the allocation: (all of it, the matrix)."""
    whole = torch.full((start + M * (N + pad),), 77.0, dtype=dtype, device="cuda")
    return whole, torch.as_strided(whole, (M, N), (N + pad, 1), start)


class Problem:
    def __init__(self, M, K, N, bw, dt, p_a=0.2, p_b=0.4, p_rows=None, seed=0, out=None, pad=0, start=0):
        self.M, self.K, self.N, self.bw, self.dt, self.out = M, K, N, bw, dt, out or dt
        g = torch.Generator().manual_seed(seed + M + K + N)
        t = T[dt][1]
        self.X, self.Y = torch.randn(M, K, generator=g).to(t).cuda(), (torch.randn(K, N, generator=g) * 0.3).to(t).cuda()
        keep = torch.rand(M, K, generator=g) < p_a
        blocks = torch.rand(K, N // bw, generator=g) < p_b
        if M > 2:
            keep[1] = False            # a row without any product
        blocks[:, 0] = False           # nor columns
        rows = None if p_rows is None else torch.rand(1, K, generator=g) < p_rows
        on = blocks if rows is None else blocks & rows.view(-1, 1)
        self.A = self.X.double().cpu() * keep
        self.B = self.Y.double().cpu() * on.repeat_interleave(bw, 1)
        self.keep, self.rows, self.blocks = words(keep), None if rows is None else words(rows), words(blocks)
        self.bias = torch.randn(N, generator=g).to(t).cuda()
        o = T[self.out][1]
        self.Rall, self.R = room(M, N, o, pad, start)
        self.R.copy_(torch.randn(M, N, generator=g).to(o))
        self.Call, self.C = room(M, N, o, pad, start)
        self.Zall, self.Z = room(M, N, o, pad, start)
        self.plain = torch.empty(M, N, dtype=torch.float64 if dt == "f64" else torch.float32, device="cuda")
        self.eng = mm.MaskedMatmul(M, K, N, bw, T[dt][0])
        self.eng.build_maps(self.X, self.Y, keep_a=self.keep, keep_rows=self.rows, keep_blocks=self.blocks)

    def expected(self, bias, act, residual):
        """The same steps behind the product, one float operation each."""
        z = self.plain + self.bias.to(self.plain.dtype) if bias else self.plain.clone()
        c = torch.where(z < 0, torch.zeros_like(z), z) if act == "relu" else z
        if residual:
            c = c + self.R.to(self.plain.dtype)
        return z.to(self.C.dtype), c.to(self.C.dtype)

    def bit_for_bit(self, what, fused=False):
        if fused:
            self.eng.matmul_fused(self.X, self.Y, self.plain, keep_a=self.keep)
        else:
            self.eng.matmul(self.X, self.Y, self.plain)
        how = dict(pred=mm.MMM_PRED_NONZERO, keep_a=self.keep) if fused else {}
        for bias, act, residual, preact in ((False, "none", False, False), (True, "relu", True, True), (True, "none", False, True), (False, "relu", True, False)):
            self.Call.fill_(77.0)
            self.Zall.fill_(77.0)
            self.eng.matmul_epilogue(self.X, self.Y, self.C, bias=self.bias if bias else None, activation=ACTS[act], residual=self.R if residual else None,
                                     preact=self.Z if preact else None, **how)
            z, c = self.expected(bias, act, residual)
            assert torch.equal(self.C, c), (what, bias, act, residual)
            assert not preact or torch.equal(self.Z, z), (what, "preact")
            for whole, t in ((self.Call, self.C), (self.Zall, self.Z)):   # what lies around it is as it was
                t.fill_(77.0)
                assert bool((whole == 77.0).all()), (what, "outside")
        self.C.copy_(self.R)          # in place: C is added to
        self.eng.matmul_epilogue(self.X, self.Y, self.C, activation=ACTS["relu"], residual=self.C, **how)
        assert torch.equal(self.C, self.expected(False, "relu", True)[1]), (what, "in place")


# every tile, K in one part and in three, both widths of lists, rows and columns that do not fill their tiles (N: half a group of 16 behind the last
# whole one), a C that begins and goes on at odd elements
@pytest.mark.gpu
@pytest.mark.parametrize("bw", [8, 16, 32])
@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f64", "f64")])
@pytest.mark.parametrize("M", [30, 130])
def test_every_tile(M, dt, out, bw):
    p = Problem(M, 700, 264 if bw == 8 else 288, bw, dt, out=out, pad=1, start=1)
    if dt == "f64" and M <= 64:
        p.bit_for_bit("pairs")
        return
    p.eng.set_path(mm.MMM_PATH_MATRIX)
    for v in range(mm.mmm_matmul_variant_count()):
        for split in (1, 3):
            p.eng.set_plan(v, split)
            got = p.eng.plan()
            if got[0] == v and got[1] == split:
                p.bit_for_bit((mm.mmm_matmul_variant_name(v), split))


@pytest.mark.gpu
@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f64", "f64")])
@pytest.mark.parametrize("M,K,N,bw", [(1, 1, 8, 8), (1, 5000, 264, 8), (7, 333, 96, 16), (70, 200, 1056, 32)])
def test_pairs_and_fused(M, K, N, bw, dt, out):
    p = Problem(M, K, N, bw, dt, out=out, p_a=0.5 if K > 1 else 1.0)
    p.eng.set_path(mm.MMM_PATH_PAIRS)
    p.bit_for_bit("pairs")
    p.bit_for_bit("fused", fused=True)


@pytest.mark.gpu
@pytest.mark.parametrize("form", [0, 1])
@pytest.mark.parametrize("bw", [8, 32])
def test_floats_in_parts_and_rows_by_context(form, bw):
    mm.mmm_set_option("float_form", form)
    try:
        for rows in (None, 0.3):
            p = Problem(200, 1100, 544, bw, "f32", p_rows=rows)
            p.eng.set_path(mm.MMM_PATH_MATRIX)
            assert mm.mmm_matmul_form(p.eng.maps) == form
            p.bit_for_bit(("form", form, rows))
    finally:
        mm.mmm_set_option("float_form", -1)
    q = Problem(200, 1100, 544, bw, "bf16", p_rows=0.3)
    q.eng.set_path(mm.MMM_PATH_MATRIX)
    q.bit_for_bit("rows")


@pytest.mark.gpu
def test_columns_left_out():
    """Floats whose columns are zero in whole tiles: the lists without them."""
    p = Problem(128, 2048, 512, 16, "f32", p_b=1.0)
    cols = torch.zeros(128, 2048, dtype=torch.bool)
    cols[:, ::9] = True
    keep = words(cols)
    p.eng.build_maps(p.X, p.Y, keep_a=keep, keep_blocks=p.blocks)
    p.eng.stats()
    p.eng.set_path(mm.MMM_PATH_MATRIX)
    for v in range(mm.mmm_matmul_variant_count()):
        p.eng.set_plan(v, 1)
        if p.eng.plan()[0] == v:
            p.bit_for_bit(("columns", v))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N,bw,dt,path", [(130, 300, 264, 8, "f32", 0), (130, 300, 264, 8, "bf16", 0), (3, 900, 96, 16, "f16", 1), (70, 300, 96, 32, "f64", 0),
                                              (33, 129, 64, 32, "f64", 1)])
def test_activations(act, M, K, N, bw, dt, path):
    p = Problem(M, K, N, bw, dt)
    p.eng.set_path(path)
    p.eng.matmul_epilogue(p.X, p.Y, p.C, bias=p.bias, activation=ACTS[act], residual=p.R, preact=p.Z)
    b, r = p.bias.double().cpu(), p.R.double().cpu()
    z, mag = p.A @ p.B + b, p.A.abs() @ p.B.abs() + b.abs()
    c = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * 0.5 * torch.erfc(-z / math.sqrt(2)),
         "gelu_tanh": lambda: z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)), "silu": lambda: z * torch.sigmoid(z)}[act]()
    half, wide = torch.finfo(p.C.dtype).eps / 2, 2.0 ** -53 if dt == "f64" else U
    sums = (1e-12 if dt == "f64" else 1e-5) * mag
    for got, want, bound in ((p.Z, z, sums), (p.C, c + r, 1.13 * sums + 16 * wide * (1 + z.abs() + r.abs()))):
        err = (got.double().cpu() - want).abs()
        bound = bound + half * want.abs() * (1 + 1e-3)
        assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["f32", "bf16", "f64"])
def test_arguments_at_the_ends(act, dt):
    """A bias that is large, infinite or NaN where there is no product: the limits of the activation."""
    values = [0.0, -0.0, 200.0, -200.0, 1e30, -1e30, float("inf"), -float("inf"), float("nan"), 1.0, -1.0, 3.0, -3.0, 40.0, -40.0, 1e-30]
    X, Y = torch.zeros(2, 8, dtype=T[dt][1], device="cuda"), torch.zeros(8, 16, dtype=T[dt][1], device="cuda")
    bias = torch.tensor(values, dtype=T[dt][1], device="cuda")
    C = torch.empty(2, 16, dtype=T[dt][1], device="cuda")
    eng = mm.MaskedMatmul(2, 8, 16, 8, T[dt][0])
    eng.build_maps(X, Y)
    eng.matmul_epilogue(X, Y, C, bias=bias, activation=ACTS[act])
    for row in C.double().cpu().tolist():
        low = 0.0 if act != "none" else None
        for got, z in zip(row, bias.double().cpu().tolist()):
            if math.isnan(z):
                assert math.isnan(got)
            elif abs(z) >= 200:
                # (a sigmoid in double is not 0 at -200: 200 e^-200 = 200 * 1.3839e-87 = 2.768e-85; in float it is, e^-88 and less leave the range)
                limit = z if z > 0 or low is None else 0.0
                assert got == limit or (dt == "f64" and z == -200 and abs(got) <= 2.769e-85), (got, z)
            elif z in (0.0, 40.0):
                assert abs(got - z) <= 40 * torch.finfo(C.dtype).eps


@pytest.mark.gpu
def test_masked_places_hold_anything():
    """NaN and infinities at masked places of X and in blocks that are off do not reach C; behind the last row and column nothing is written."""
    p = Problem(70, 300, 96, 16, "bf16")
    p.eng.build_maps(p.X, p.Y, keep_a=p.keep, keep_blocks=p.blocks)
    p.eng.matmul_epilogue(p.X, p.Y, p.C, bias=p.bias, activation=ACTS["gelu"])
    X, Y = p.X.clone(), p.Y.clone()
    X[(p.A == 0).cuda()] = float("nan")
    Y[(p.B == 0).cuda()] = float("inf")
    p.eng.build_maps(X, Y, keep_a=p.keep, keep_blocks=p.blocks)
    C = torch.empty_like(p.C)
    p.eng.matmul_epilogue(X, Y, C, bias=p.bias, activation=ACTS["gelu"])
    assert torch.equal(C, p.C)


@pytest.mark.gpu
@pytest.mark.parametrize("M,path,split", [(130, 0, 1), (130, 0, 3), (4, 1, 1)])
def test_another_stream_and_a_replayed_graph(M, path, split):
    p = Problem(M, 900, 96, 16, "bf16")
    p.eng.set_path(path)
    p.eng.set_plan(-1, split)

    def call(C):
        p.eng.build_maps(p.X, None, keep_a=p.keep)
        p.eng.matmul_epilogue(p.X, p.Y, C, bias=p.bias, activation=ACTS["silu"], residual=p.R)
    call(p.C)
    want = p.C.clone()
    torch.cuda.synchronize()
    side, C = torch.cuda.Stream(), torch.empty_like(want)
    with torch.cuda.stream(side):
        call(C)
    side.synchronize()
    assert torch.equal(C, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(C)
    for _ in range(3):
        C.fill_(0.0)
        call(p.C)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, want) and torch.equal(p.C, want)


# Roundings that count, each 2^-24 / sqrt 3 of the result in the mean square at most: GELU the last sum, the bell and the tail; SiLU also a reciprocal; the tanh form
# also its argument.  Their squares add up.
@pytest.mark.gpu
@pytest.mark.parametrize("act,roundings", [("gelu", 3), ("silu", 4), ("gelu_tanh", 5)])
def test_smooth_activations_of_floats_in_the_mean(act, roundings):
    """A million arguments of a layer's distribution: activation and slope by the 2-norm, in floats."""
    g = torch.Generator(device="cuda").manual_seed(6)
    M, N = 1000, 1000
    z = torch.randn(M, N, generator=g, device="cuda") - 0.5
    X, Y = torch.zeros(1, 8, device="cuda"), torch.zeros(8, N, device="cuda")
    C, dZ, ones = torch.empty_like(z), torch.empty_like(z), torch.ones_like(z)
    # the argument comes in as the bias of a row at a time
    row = mm.MaskedMatmul(1, 8, N, 8, mm.MMM_F32)
    row.build_maps(X, Y)
    for i in range(M):
        row.matmul_epilogue(X, Y, C[i:i + 1], bias=z[i], activation=ACTS[act])
    mm.mmm_epilogue_backward(M, N, mm.MMM_F32, mm.MMM_F32, ACTS[act], ones, N, z, N, dZ, N)
    d = z.double()
    if act == "gelu":
        p = 0.5 * torch.erfc(-d / math.sqrt(2))
        want, slope = d * p, p + d * torch.exp(-0.5 * d * d) / math.sqrt(2 * math.pi)
    else:
        inner, inner_slope = (d, 1.0) if act == "silu" else (math.sqrt(8 / math.pi) * (d + 0.044715 * d ** 3), math.sqrt(8 / math.pi) * (1 + 0.134145 * d ** 2))
        p = torch.sigmoid(inner)
        want, slope = d * p, p + d * p * torch.sigmoid(-inner) * inner_slope
    errors = [float((got.double() - w).norm() / w.norm()) for got, w in ((C, want), (dZ, slope))]
    print(act, errors)
    assert max(errors) <= math.sqrt(roundings / 3) * U, errors


@pytest.mark.gpu
def test_columns_left_out_are_not_multiplied():
    """What rows of Y hold whose column of A is zero in a whole tile: a kernel that multiplied them by their zeros would bring NaN."""
    M, K, N = 128, 2048, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    X, Y = torch.randn(M, K, generator=g, device="cuda"), torch.randn(K, N, generator=g, device="cuda")
    X[:, torch.arange(K, device="cuda") % 9 != 0] = 0.0
    bias, R = torch.randn(N, generator=g, device="cuda"), torch.randn(M, N, generator=g, device="cuda")
    dirty = Y.clone()
    dirty[torch.arange(K, device="cuda") % 9 != 0, ::3] = float("nan")
    eng = mm.MaskedMatmul(M, K, N, 16, mm.MMM_F32)
    eng.set_path(mm.MMM_PATH_MATRIX)
    eng.build_maps(X, Y)
    eng.stats()
    tiles = []
    for v in range(mm.mmm_matmul_variant_count()):
        eng.set_plan(v, 1)
        if eng.plan()[:2] != (v, 1):
            continue
        outs = []
        for right in (Y, dirty):
            eng.build_maps(X, right)
            assert mm.mmm_matmul_form(eng.maps) == 0
            C = torch.empty(M, N, device="cuda")
            eng.matmul_epilogue(X, right, C, bias=bias, activation=ACTS["relu"], residual=R)
            outs.append(C)
        assert bool(outs[0].isfinite().all()) and torch.equal(*outs), v
        tiles.append(v)
    assert tiles == [0, 1, 2, 6, 7]
