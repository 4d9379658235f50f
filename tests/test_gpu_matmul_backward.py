"""The gradients of the masked product against the formulas in 64 bits, under the maps as built.

Bound: a float sum of n products of exact operands is off by at most n roundings of 2^-24 of the sum of their magnitudes, whatever the order
(floats: and one for the product); n is the length of the contraction here.  dX is rounded to its type once more.  Small whole numbers are exact."""
import pytest
import torch

import paper_2402_14118_amd as mm
from test_gpu_matmul_epilogue import T, room, words

U = 2.0 ** -24


class Problem:
    def __init__(self, M, K, N, bw, dt, p_a=0.3, p_b=0.5, p_rows=None, pad=0, whole=False, seed=0):
        self.M, self.K, self.N, self.bw, self.dt = M, K, N, bw, dt
        g = torch.Generator().manual_seed(seed + 3 * M + 5 * K + 7 * N)
        t = T[dt][1]

        def values(r, c):
            v = torch.randint(-3, 4, (r, c), generator=g).float() if whole else torch.randn(r, c, generator=g)
            return v.to(t)
        X, Y, dC = values(M, K), values(K, N), values(M, N)
        keep = torch.rand(M, K, generator=g) < p_a
        blocks = torch.rand(K, N // bw, generator=g) < p_b
        if M > 3:
            keep[2] = False
        if K > 3:
            blocks[1] = False
        rows = None if p_rows is None else torch.rand(1, K, generator=g) < p_rows
        on = (blocks if rows is None else blocks & rows.view(-1, 1)) & (Y.view(K, -1, bw) != 0).any(2)
        self.a_on, self.b_on = keep & (X != 0), on.repeat_interleave(bw, 1)
        self.A, self.B, self.G = X.double() * self.a_on, Y.double() * self.b_on, dC.double()
        # what is masked out may hold anything
        X[~keep] = float("nan")
        Y[~(blocks if rows is None else blocks & rows.view(-1, 1)).repeat_interleave(bw, 1)] = float("inf")
        self.X, self.Y, self.dC = (room(*v.shape, t, pad, 1 if pad else 0)[1].copy_(v.cuda()) for v in (X, Y, dC))
        self.dXall, self.dX = room(M, K, t, pad, 1 if pad else 0)
        self.dYall, self.dY = room(K, N, torch.float32, pad, 1 if pad else 0)
        self.eng = mm.MaskedMatmul(M, K, N, bw, T[dt][0])
        self.eng.build_maps(self.X, self.Y, keep_a=words(keep), keep_rows=None if rows is None else words(rows), keep_blocks=words(blocks))

    def check(self, exact=False):
        self.dXall.fill_(77.0)
        self.dYall.fill_(77.0)
        self.eng.matmul_backward(self.X, self.Y, self.dC, self.dX, self.dY)
        half = torch.finfo(self.dX.dtype).eps / 2
        want = (self.G @ self.B.t()) * self.a_on, (self.A.t() @ self.G) * self.b_on
        mags = self.G.abs() @ self.B.abs().t(), self.A.abs().t() @ self.G.abs()
        for what, got, w, mag, n, step in (("dX", self.dX, want[0], mags[0], self.N, half), ("dY", self.dY, want[1], mags[1], self.M, 0.0)):
            err = (got.double().cpu() - w).abs()
            bound = torch.zeros_like(err) if exact else (n + 1) * U * mag + step * w.abs() * (1 + 1e-3)
            if exact and self.dt != "f32" and what == "dX":
                bound = step * w.abs()
            assert bool((err <= bound).all()), (what, float(err.max()), int((~(err <= bound)).sum()))
        assert bool((self.dX.cpu()[~self.a_on] == 0).all()) and bool((self.dY.cpu()[~self.b_on] == 0).all())
        first, sums = self.dX.clone(), self.dY.clone()
        # added to; one of the two alone; the same again
        self.dY.fill_(1.0)
        self.eng.matmul_backward(self.X, self.Y, self.dC, dY=self.dY, accumulate=True)
        assert torch.equal(self.dY, sums + 1.0)
        self.dX.fill_(5.0)
        self.eng.matmul_backward(self.X, self.Y, self.dC, dX=self.dX)
        assert torch.equal(self.dX, first)
        self.dX.fill_(5.0)          # at every element
        self.eng.matmul_backward(self.X, self.Y, self.dC, dX=self.dX, all_x=True)
        all_dx = self.G @ self.B.t()
        assert bool(((self.dX.double().cpu() - all_dx).abs() <= (self.N + 1) * U * mags[0] + half * all_dx.abs() * (1 + 1e-3)).all())
        assert torch.equal(self.dX.cpu()[self.a_on], first.cpu()[self.a_on])
        for whole, t in ((self.dXall, self.dX), (self.dYall, self.dY)):
            t.fill_(77.0)
            assert bool((whole == 77.0).all()), "outside"


SHAPES = [(1, 1, 8, 8), (3, 7, 16, 16), (17, 130, 40, 8), (64, 128, 128, 16), (65, 129, 136, 8), (200, 333, 264, 8), (129, 1000, 160, 32), (300, 257, 1056, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [None, 0.3])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K,N,bw", SHAPES)
def test_gradients(M, K, N, bw, dt, rows):
    Problem(M, K, N, bw, dt, p_rows=rows, pad=3 if M % 2 else 0).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_whole_numbers_are_exact(dt):
    Problem(150, 300, 200, 8, dt, whole=True).check(exact=True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [None, 0.4])
def test_floats_in_parts(rows):
    """The image of A in three parts, among them elements that parts do not hold."""
    mm.mmm_set_option("float_form", 1)
    try:
        p = Problem(200, 300, 264, 8, "f32", p_rows=rows)
        assert mm.mmm_matmul_form(p.eng.maps) == 1
        p.check()
        at = p.a_on.nonzero()[5]
        X = p.X.clone()
        X[at[0], at[1]] = 2.0 ** 60
        p.A[at[0], at[1]] = 2.0 ** 60
        p.eng.build_maps(X, None, keep_a=words(p.a_on))
        p.X = X
        p.check()
    finally:
        mm.mmm_set_option("float_form", -1)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("p_rows", [0.0, 1.0])
def test_all_or_none(dt, p_rows):
    """No live row at all (both gradients are zero), and all of them."""
    Problem(70, 200, 64, 16, dt, p_rows=p_rows).check()
    Problem(70, 200, 64, 16, dt, p_a=0.0).check()
    Problem(70, 200, 64, 16, dt, p_a=1.0, p_b=1.0).check()


@pytest.mark.gpu
def test_gradients_against_differences():
    """Along random directions of the kept elements the product is linear in each operand: C(X + e) - C(X) is the slope itself but for rounding, 300
    roundings of 2^-24 of the sum of magnitudes."""
    p = Problem(40, 300, 96, 16, "f32")
    p.eng.matmul_backward(p.X, p.Y, p.dC, p.dX, p.dY)
    g = torch.Generator().manual_seed(3)
    wx, wy = torch.randn(40, 300, generator=g).double() * p.a_on, torch.randn(300, 96, generator=g).double() * p.b_on
    for grad, along, change in ((p.dX, wx, wx @ p.B), (p.dY, wy, p.A @ wy)):
        terms = grad.double().cpu() * along
        assert abs(float((p.G * change).sum()) - float(terms.sum())) <= 300 * U * float((p.G.abs() @ p.B.abs().t() * along.abs()).sum() if grad is p.dX
                                                                                      else (p.A.abs().t() @ p.G.abs() * along.abs()).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [None, 0.3])
def test_another_stream_and_a_replayed_graph(rows):
    p = Problem(130, 400, 200, 8, "bf16", p_rows=rows)
    p.eng.matmul_backward(p.X, p.Y, p.dC, p.dX, p.dY)
    want = p.dX.clone(), p.dY.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        p.dX.fill_(3.0)
        p.dY.fill_(3.0)
        p.eng.matmul_backward(p.X, p.Y, p.dC, p.dX, p.dY)
    side.synchronize()
    assert torch.equal(p.dX, want[0]) and torch.equal(p.dY, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.eng.matmul_backward(p.X, p.Y, p.dC, p.dX, p.dY)
    for _ in range(3):
        p.dX.fill_(3.0)
        p.dY.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.dX, want[0]) and torch.equal(p.dY, want[1])


# sizes whose results fill 128 x 128 and 256 x 256 tiles (and the edges of them), and long contractions over few results, whose parts are joined
@pytest.mark.gpu
@pytest.mark.parametrize("dt,M,K,N,rows", [("bf16", 1000, 4100, 2080, None), ("f16", 2048, 2048, 1032, 0.5), ("f32", 1300, 2300, 1544, None), ("f32", 2050, 3000, 1032, 0.4),
                                           ("bf16", 2900, 5000, 4104, None), ("bf16", 24, 70, 8192, None), ("f32", 2048, 72, 136, None), ("f16", 2000, 130, 64, 0.5)])
def test_tiles_and_parts(dt, M, K, N, rows):
    """The reference on the device, in 64 bits: the sizes are larger here."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    t = T[dt][1]
    X, Y, dC = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((M, K), (K, N), (M, N)))
    keep = torch.rand(M, K, generator=g, device="cuda") < 0.3
    blocks = torch.rand(K, N // 8, generator=g, device="cuda") < 0.5
    on_rows = None if rows is None else torch.rand(1, K, generator=g, device="cuda") < rows
    eng = mm.MaskedMatmul(M, K, N, 8, T[dt][0])
    eng.build_maps(X, Y, keep_a=words(keep.cpu()), keep_rows=None if rows is None else words(on_rows.cpu()), keep_blocks=words(blocks.cpu()))
    a_on = keep & (X != 0)
    b_on = (blocks if rows is None else blocks & on_rows.view(-1, 1)).repeat_interleave(8, 1)
    A, Bm, G = X.double() * a_on, Y.double() * b_on, dC.double()
    half = torch.finfo(t).eps / 2
    for counted in (False, True):
        if counted:
            eng.stats()   # (the number of live rows is then known to the choice of tile)
        dX, dY = torch.full_like(X, 7.0), torch.full((K, N), 7.0, device="cuda")
        eng.matmul_backward(X, Y, dC, dX, dY)
        for got, want, mag, n, step in ((dX, (G @ Bm.t().contiguous()) * a_on, G.abs() @ Bm.abs().t().contiguous(), N, half),
                                        (dY, (A.t().contiguous() @ G) * b_on, A.abs().t().contiguous() @ G.abs(), M, 0.0)):
            assert bool(((got.double() - want).abs() <= (n + 1) * U * mag + step * want.abs() * (1 + 1e-3)).all())
        more = dY.clone()
        eng.matmul_backward(X, Y, dC, dY=more, accumulate=True)
        assert torch.equal(more, dY + dY)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_captured_step_with_another_selection(dt):
    """The maps are made again inside a graph: replays follow the rows selected then, of which there may be far more than when it was captured."""
    M, K, N = 200, 3000, 264
    g = torch.Generator().manual_seed(5)
    t = T[dt][1]
    X, Y, dC = (torch.randn(s, generator=g).to(t).cuda() for s in ((M, K), (K, N), (M, N)))
    few, many = (words(torch.rand(1, K, generator=g) < p) for p in (0.02, 0.95))
    chosen = few.clone()
    eng = mm.MaskedMatmul(M, K, N, 8, T[dt][0])
    dX, dY = torch.empty_like(X), torch.empty(K, N, device="cuda")

    def call():
        eng.build_maps(X, Y, keep_rows=chosen)
        eng.matmul_backward(X, Y, dC, dX, dY)
    call()
    eng.stats()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rows in (many, few, many, torch.zeros_like(few)):
        chosen.copy_(rows)
        dX.fill_(3.0)
        dY.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        bits = (rows.view(torch.uint8).cpu().view(-1, 1) >> torch.arange(8, dtype=torch.uint8) & 1).reshape(-1)[:K].bool().cuda()
        B, A, G = Y.double() * bits.view(-1, 1), X.double(), dC.double()
        a_on = (X != 0)
        want, mag = (G @ B.t().contiguous()) * a_on, G.abs() @ B.abs().t().contiguous()
        assert bool(((dX.double() - want).abs() <= (N + 1) * U * mag + torch.finfo(t).eps / 2 * want.abs() * (1 + 1e-3)).all())
        want, mag = (A.t().contiguous() @ G) * bits.view(-1, 1), A.abs().t().contiguous() @ G.abs()
        assert bool(((dY.double() - want).abs() <= (M + 1) * U * mag).all())


@pytest.mark.gpu
def test_rows_far_apart():
    """Leading dimensions next to the largest: offsets of rows pass 32 bits."""
    M, K, N, ld = 1100, 1030, 64, (1 << 22) - 8
    g = torch.Generator().manual_seed(9)
    host = [torch.randn(s, generator=g).bfloat16() for s in ((M, K), (K, N), (M, N))]
    near = [v.cuda() for v in host]
    far = [torch.empty(v.shape[0] * ld, dtype=v.dtype, device="cuda").as_strided(v.shape, (ld, 1)).copy_(v) for v in near]
    results = []
    for (X, Y, dC), pitch in ((near, None), (far, ld)):
        eng = mm.MaskedMatmul(M, K, N, 8, mm.MMM_BF16)
        eng.build_maps(X, Y)
        room = lambda v, t: torch.empty(v.shape, dtype=t, device="cuda") if pitch is None else torch.empty(v.shape[0] * pitch, dtype=t, device="cuda").as_strided(v.shape, (pitch, 1))
        dX, dY, C = room(X, X.dtype), room(Y, torch.float32), room(dC, dC.dtype)
        eng.matmul_backward(X, Y, dC, dX, dY)
        eng.matmul_epilogue(X, Y, C, activation=mm.MMM_ACT_SILU, residual=dC)
        results.append([v.clone(memory_format=torch.contiguous_format) for v in (dX, dY, C)])
        eng.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))


# 16-bit results of many tiles with rows by context: dX is written in whole rows, each tile from its first live row of B to the next tile's
@pytest.mark.gpu
@pytest.mark.parametrize("dt,M,K,N,which", [("bf16", 2051, 2055, 72, "none"), ("f16", 2051, 2055, 72, "first"), ("bf16", 2051, 2055, 72, "last"), ("f16", 2100, 2055, 72, "middle"),
                                            ("bf16", 2051, 2055, 72, 0.1), ("f16", 4001, 1153, 136, 0.5), ("bf16", 1030, 8200, 520, 0.5), ("f16", 2051, 16391, 1032, 0.9),
                                            ("bf16", 2051, 16391, 264, "ends")])
def test_whole_rows(dt, M, K, N, which):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    t = T[dt][1]
    X, Y, dC = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((M, K), (K, N), (M, N)))
    keep = torch.rand(M, K, generator=g, device="cuda") < 0.4
    on = torch.rand(K, generator=g, device="cuda") < (which if isinstance(which, float) else 0.0)
    if which == "first":
        on[0] = True
    if which == "last":
        on[K - 1] = True
    if which == "middle":
        on[700:1400] = True
    if which == "ends":
        on[:300] = True
        on[-1400:] = True
    eng = mm.MaskedMatmul(M, K, N, 8, T[dt][0])
    eng.build_maps(X, Y, keep_a=words(keep.cpu()), keep_rows=words(on.view(1, -1).cpu()))
    a_on = keep & (X != 0)
    Bm, G = Y.double() * on.view(-1, 1), dC.double()
    want, mag = G @ Bm.t().contiguous(), G.abs() @ Bm.abs().t().contiguous()
    whole, dX = room(M, K, t, 3, 1)
    for counted in (False, True):
        if counted:
            eng.stats()   # (then a selection of few rows is known as such)
        for all_x in (False, True):
            whole.fill_(77.0)
            eng.matmul_backward(X, Y, dC, dX, all_x=all_x)
            w = want if all_x else want * a_on
            assert bool(((dX.double() - w).abs() <= (N + 1) * U * mag + torch.finfo(t).eps / 2 * w.abs() * (1 + 1e-3)).all()), (counted, all_x)
            assert bool((dX[:, ~on] == 0).all()) and (all_x or bool((dX[~a_on] == 0).all()))
            dX.fill_(77.0)
            assert bool((whole == 77.0).all()), "outside"


@pytest.mark.gpu
@pytest.mark.parametrize("form", [0, 1])
def test_a_captured_gradient_fixes_the_form(form):
    """dY of a graph reads the image of A as it was laid out when it was captured: builds that follow keep to that, whatever they would choose."""
    try:
        mm.mmm_set_option("float_form", form)
        p = Problem(150, 300, 200, 8, "f32", whole=True)
        keep, blocks = words(p.a_on), words(p.b_on[:, ::8])
        p.check(exact=True)
        want = p.A.t() @ p.G * p.b_on
        p.dYall.fill_(77.0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.eng.matmul_backward(p.X, p.Y, p.dC, dY=p.dY)
        mm.mmm_set_option("float_form", 1 - form)
        p.eng.stats()
        for _ in range(3):
            p.eng.build_maps(p.X, p.Y, keep_a=keep, keep_blocks=blocks)
            assert mm.mmm_matmul_form(p.eng.maps) == form
            p.dY.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.dY.double().cpu(), want)
            p.check(exact=True)
    finally:
        mm.mmm_set_option("float_form", -1)


TILES = [("bf16", 1000, 4100, 2080, None), ("f16", 2048, 2048, 1032, 0.5), ("f32", 1300, 2300, 1544, None), ("f32", 2050, 3000, 1032, 0.4), ("bf16", 2900, 5000, 4104, None),
         ("bf16", 24, 70, 8192, None), ("f32", 2048, 72, 136, None), ("f16", 2000, 130, 64, 0.5), ("bf16", 2051, 2055, 72, 0.1), ("f16", 4001, 1153, 136, 0.5),
         ("bf16", 1030, 8200, 520, 0.5), ("f16", 2051, 16391, 1032, 0.9), ("f32", 777, 3001, 1992, 0.25)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt,M,K,N,rows", TILES)
def test_whole_numbers_in_every_tile(dt, M, K, N, rows):
    """All tiles, parts and ways of storing, with whole numbers from -3 to 3: sums are exact (9 * 8192 < 2^24), so a product that is lost or counted twice shows."""
    g = torch.Generator(device="cuda").manual_seed(M + K + N)
    t = T[dt][1]
    X, Y, dC = (torch.randint(-3, 4, s, generator=g, device="cuda").to(t) for s in ((M, K), (K, N), (M, N)))
    keep = torch.rand(M, K, generator=g, device="cuda") < 0.6
    blocks = torch.rand(K, N // 8, generator=g, device="cuda") < 0.7
    on = torch.ones(K, dtype=torch.bool, device="cuda") if rows is None else torch.rand(K, generator=g, device="cuda") < rows
    eng = mm.MaskedMatmul(M, K, N, 8, T[dt][0])
    eng.build_maps(X, Y, keep_a=words(keep.cpu()), keep_rows=None if rows is None else words(on.view(1, -1).cpu()), keep_blocks=words(blocks.cpu()))
    A, Bm, G = X.double() * keep, Y.double() * (blocks & on.view(-1, 1)).repeat_interleave(8, 1), dC.double()
    all_dx, want_y = G @ Bm.t().contiguous(), (A.t().contiguous() @ G) * (Bm.view(K, -1, 8) != 0).any(2).repeat_interleave(8, 1)
    for counted in (False, True):
        if counted:
            eng.stats()
        dX, dY = torch.full_like(X, 7.0), torch.full((K, N), 7.0, device="cuda")
        eng.matmul_backward(X, Y, dC, dX, dY)
        assert torch.equal(dX, (all_dx * (A != 0)).to(t)) and torch.equal(dY.double(), want_y), counted
        eng.matmul_backward(X, Y, dC, dX, all_x=True)
        assert torch.equal(dX, all_dx.to(t)), counted
