"""The operators together: a residual MLP block, forward and backward, against the same block in 64 bits and its automatic differentiation.

Floats.  Each of the eight steps errs by at most 130 roundings of 2^-24 (sums of at most 128 terms) of the magnitudes it adds, 7.8e-6; the
magnitudes are up to sqrt(128) times the results (random signs): 8 * 7.8e-6 * 12 = 7.5e-4 of the largest value of an output at most.  No argument
of ReLU lies within 1e-4 of zero, so that no error turns a unit on or off.  bf16: a step rounds its output by 2^-9 at most; eight of them,
amplified the same, stay below .19 of the largest value; the 2-norm, where they add up as random numbers, below .05."""
import pytest
import torch

import paper_2402_14118_amd as mm
from test_gpu_block_norm import standard as rows_standard
from test_gpu_matmul_epilogue import T, words

EPS = 1e-5


def standard(x, layer):
    x = x - x.mean(1, keepdim=True) if layer else x
    return x / (x.pow(2).mean(1, keepdim=True) + EPS).sqrt()


def block(p, act, on1, on2):
    a = p["N"] @ (p["W1"] * on1) + p["b1"]
    z = a
    a = {"relu": torch.relu, "silu": torch.nn.functional.silu}[act](a)
    y = a @ (p["W2"] * on2) + p["b2"]
    h = 0.9 * p["H"] + p["gate"] * (standard(y, False) * p["post_weight"])
    return z, h, standard(h, True) * p["pre_weight"] + p["pre_bias"]


def setup(dt, act, M=40, d=64, f=128, context=True, **how):
    g = torch.Generator().manual_seed(11)
    t = T[dt][1]
    shapes = dict(N=((M, d), 1.0, 0.0), W1=((d, f), 0.15, 0.0), b1=((f,), 0.3, -0.5), W2=((f, d), 0.1, 0.0), b2=((d,), 0.1, 0.0), H=((M, d), 1.0, 0.0),
                  gate=((d,), 0.3, 0.5), post_weight=((d,), 0.1, 1.0), pre_weight=((d,), 0.1, 1.0), pre_bias=((d,), 0.1, 0.0))
    host = {k: (torch.randn(s, generator=g) * std + mean).to(t) for k, (s, std, mean) in shapes.items()}
    k1, k2, r2 = torch.rand(d, f // 16, generator=g) < 0.7, torch.rand(f, d // 16, generator=g) < 0.8, torch.rand(1, f, generator=g) < 0.5
    on1 = k1.repeat_interleave(16, 1)
    on2 = k2.repeat_interleave(16, 1) & (r2.view(-1, 1) if context else True)
    dev = {k: v.cuda() for k, v in host.items()}
    mlp = mm.MaskedMlp(M, d, f, 16, T[dt][0], mm.MMM_ACT_RELU if act == "relu" else mm.MMM_ACT_SILU, mm.MMM_NORM_RMS, mm.MMM_NORM_LAYER, mm.MMM_GATE_COL, 0.9, EPS, **how)
    mlp.set_weights(dev["W1"], dev["W2"], dev["b1"], dev["b2"], words(k1), words(k2), words(r2) if context else None)
    return mlp, dev, {k: v.double().requires_grad_() for k, v in host.items()}, on1.double(), on2.double()


def close(got, want, dt, what):
    err = (got.double().cpu() - want).abs()
    limit = (7.5e-4 if dt == "f32" else 0.19) * float(want.abs().max())
    assert float(err.max()) <= limit, (what, float(err.max()), limit)
    if dt != "f32":
        assert float(err.norm()) <= 0.05 * float(want.norm()), (what, float(err.norm() / want.norm()))


@pytest.mark.gpu
@pytest.mark.parametrize("dt,act,context", [("f32", "relu", True), ("f32", "silu", False), ("bf16", "silu", True), ("f16", "relu", False)])
def test_training_step(dt, act, context):
    mlp, d, ref, on1, on2 = setup(dt, act, context=context, training=True)
    values = {k: d[k] for k in ("gate", "post_weight", "pre_weight")}
    H_out, n = torch.empty_like(d["H"]), torch.empty_like(d["H"])
    mlp.forward(d["N"], d["H"], H_out, n, pre_bias=d["pre_bias"], **values)
    z, h, want_n = block(ref, act, on1, on2)
    if act == "relu" and dt == "f32":
        assert float(z.detach().abs().min()) > 1e-4
    close(H_out, h.detach(), dt, "H_out")
    close(n, want_n.detach(), dt, "n")
    g = torch.Generator().manual_seed(4)
    up_n, up_h = (torch.randn(h.shape, generator=g).to(T[dt][1]) for _ in range(2))
    ((want_n * up_n.double()).sum() + (h * up_h.double()).sum()).backward()

    def grads():
        out = {"grad_N": torch.empty_like(d["N"]), "grad_H": torch.empty_like(d["H"]), **{"grad_" + k: torch.full(d[k].shape, float("nan"), device="cuda")
               for k in ("W1", "W2", "b1", "b2", "gate", "post_weight", "pre_weight", "pre_bias")}}
        mlp.backward(d["N"], H_out, grad_normed=up_n.cuda(), grad_H_out=up_h.cuda(), **values, **out)
        return out
    out = grads()
    for k, v in out.items():
        close(v, ref[k[5:]].grad, dt, k)
    # a step captured into a graph, replayed with the program's own step between replays
    torch.cuda.synchronize()
    un, uh = up_n.cuda(), up_h.cuda()
    again = {k: torch.empty_like(v) for k, v in out.items()}
    H2, n2 = torch.empty_like(H_out), torch.empty_like(n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp.forward(d["N"], d["H"], H2, n2, pre_bias=d["pre_bias"], **values)
        mlp.backward(d["N"], H2, grad_normed=un, grad_H_out=uh, **values, **again)
    for _ in range(3):
        for t in (H2, n2, *again.values()):
            t.fill_(0.0)
        mlp.forward(d["N"], d["H"], H_out, n, pre_bias=d["pre_bias"], **values)
        eager = grads()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(H2, H_out) and torch.equal(n2, n)
        assert all(torch.equal(eager[k], again[k]) and torch.equal(eager[k], out[k]) for k in out)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5])
def test_decode(M):
    """Few rows: the mask evaluated inside the second product, the stream in place and in float beside 16-bit weights."""
    mlp, d, ref, on1, on2 = setup("bf16", "relu", M=M, context=False, fused=True, dtype_h=mm.MMM_F32)
    stream, n = d["H"].float(), torch.empty_like(d["N"])
    mlp.forward(d["N"], stream, stream, n, gate=d["gate"], post_weight=d["post_weight"], pre_weight=d["pre_weight"], pre_bias=d["pre_bias"])
    _, h, want_n = block(ref, "relu", on1, on2)
    close(stream, h.detach(), "bf16", "H_out")
    close(n, want_n.detach(), "bf16", "n")


@pytest.mark.gpu
def test_order_of_calls():
    mlp, d, *_ = setup("bf16", "relu")
    out = torch.empty_like(d["H"])
    with pytest.raises(ValueError):
        mlp.backward(d["N"], out, out, out)
    with pytest.raises(ValueError):
        mm.MaskedMlp(4, 64, 64, fused=True, training=True)
    with pytest.raises(ValueError):
        mm.MaskedMlp(4, 64, 64, fused=True, activation=mm.MMM_ACT_SILU)
    with pytest.raises(ValueError):
        mm.MaskedMlp(4, 64, 64).forward(d["N"][:4], d["H"][:4], out[:4])


@pytest.mark.gpu
def test_counted():
    """After count() floats may come in parts and another kernel may run: the same block within the bounds."""
    mlp, d, ref, on1, on2 = setup("f32", "relu", M=300, d=512, f=1024, context=False)
    values = {k: d[k] for k in ("gate", "post_weight", "pre_weight", "pre_bias")}
    first, second, n = torch.empty_like(d["H"]), torch.empty_like(d["H"]), torch.empty_like(d["H"])
    mlp.forward(d["N"], d["H"], first, n, **values)
    up, down = mlp.count()
    a = torch.relu(ref["N"].detach() @ (ref["W1"].detach() * on1) + ref["b1"].detach())
    assert up[0] == int((d["N"] != 0).sum()) and abs(down[0] - int((a > 0).sum())) <= 4      # (a unit whose argument is next to zero)
    mlp.set_weights(d["W1"], d["W2"], d["b1"], d["b2"])
    mlp.forward(d["N"], d["H"], first, n, **values)
    mlp.count()
    mlp.forward(d["N"], d["H"], second, n, **values)
    close(second, first.double().cpu(), "f32", "H_out")


@pytest.mark.gpu
@pytest.mark.parametrize("M,fused", [(5, True), (5, False), (40, False)])
def test_nan_reaches_the_stream(M, fused):
    """A row that is not a number stays one behind ReLU and its mask, and touches no other."""
    mlp, d, *_ = setup("bf16", "relu", M=M, context=False, fused=fused)
    values = {k: d[k] for k in ("gate", "post_weight", "pre_weight", "pre_bias")}
    want, got, n = torch.empty_like(d["H"]), torch.empty_like(d["H"]), torch.empty_like(d["H"])
    mlp.forward(d["N"], d["H"], want, n, **values)
    assert bool(want.isfinite().all())
    d["N"][3, 7] = float("nan")
    mlp.forward(d["N"], d["H"], got, n, **values)
    others = [i for i in range(M) if i != 3]
    assert bool(got[3].isnan().all()) and bool(n[3].isnan().all()) and torch.equal(got[others], want[others])


@pytest.mark.gpu
def test_two_blocks_at_once():
    """A holder each, on streams of their own, give what they give one after the other."""
    blocks = [setup(dt, act, M=300, d=256, f=512, context=False)[:2] for dt, act in (("bf16", "relu"), ("f32", "silu"))]
    wants, gots, streams = [], [], [torch.cuda.Stream() for _ in blocks]

    def call(mlp, d, out):
        mlp.forward(d["N"], d["H"], *out, **{k: d[k] for k in ("gate", "post_weight", "pre_weight", "pre_bias")})
    for mlp, d in blocks:
        wants.append((torch.empty_like(d["H"]), torch.empty_like(d["H"])))
        gots.append([(torch.zeros_like(d["H"]), torch.zeros_like(d["H"])) for _ in range(4)])
        call(mlp, d, wants[-1])
    torch.cuda.synchronize()
    for i in range(4):
        for (mlp, d), out, s in zip(blocks, gots, streams):
            with torch.cuda.stream(s):
                call(mlp, d, out[i])
    torch.cuda.synchronize()
    for want, out in zip(wants, gots):
        assert all(torch.equal(a, b) for pair in out for a, b in zip(want, pair))


def whole_block(M=2048, d=2048, f=2048, **how):
    """A block of floats whose products are exact in any order and form: whole numbers, whose sums stay below 2^24 (|a| <= 9 d + 3, |y| <= (9 d + 3) f, but for
    signs that do not all agree: counted below)."""
    g = torch.Generator().manual_seed(2)
    N, W1, W2 = (torch.randint(-3, 4, s, generator=g).float() for s in ((M, d), (d, f), (f, d)))
    b1, b2 = torch.randint(-3, 4, (f,), generator=g).float(), torch.randint(-3, 4, (d,), generator=g).float()
    H = torch.randn(M, d, generator=g)
    most = torch.relu(N.cuda() @ W1.cuda() + b1.cuda()) @ W2.cuda().abs()
    assert float(most.max()) < 2 ** 24
    dev = [v.cuda() for v in (N, W1, W2, b1, b2, H)]
    keep = words(torch.rand(d, f // 16, generator=g) < 0.4)
    mlp = mm.MaskedMlp(M, d, f, 16, mm.MMM_F32, **how)
    mlp.set_weights(*dev[1:5], keep_blocks1=keep)
    return mlp, dev, keep


@pytest.mark.gpu
def test_the_form_of_floats_follows_the_counts():
    mlp, (N, W1, W2, b1, b2, H), keep = whole_block()
    like = mm.MaskedMatmul(2048, 2048, 2048, 16, mm.MMM_F32)
    like.set_path(mm.MMM_PATH_MATRIX)
    like.build_maps(N, W1, keep_blocks=keep)
    like.stats()
    like.build_maps(N, W1, keep_blocks=keep)
    chosen = mm.mmm_matmul_form(like.maps)
    assert chosen == 1               # (where both sides are built with the counts known)
    outs = [torch.empty_like(H) for _ in range(4)]
    n = torch.empty_like(H)
    mlp.forward(N, H, outs[0], n)
    assert mm.mmm_matmul_form(mlp.up.maps) == 0
    mlp.count()
    for out in outs[1:3]:
        mlp.forward(N, H, out, n)
        assert mm.mmm_matmul_form(mlp.up.maps) == chosen
    mlp.set_weights(W1, W2, b1, b2, keep)
    mlp.forward(N, H, outs[3], n)
    assert mm.mmm_matmul_form(mlp.up.maps) == chosen
    assert all(torch.equal(out, outs[0]) for out in outs[1:])


@pytest.mark.gpu
def test_a_captured_block_keeps_the_form_it_has():
    """Counted and captured before the next call of the program's own: the weights are not built inside the graph, and stay in its form as long as it is there."""
    mlp, (N, W1, W2, b1, b2, H), _ = whole_block()
    want, own, out, n = (torch.empty_like(H) for _ in range(4))
    mlp.forward(N, H, want, n)
    mlp.count()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp.forward(N, H, out, n)
    for _ in range(3):
        out.fill_(0.0)
        own.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        mlp.forward(N, H, own, n)
        assert mm.mmm_matmul_form(mlp.up.maps) == 0 and torch.equal(own, want)


# Each step of the block from what the step before has left in its 16 bits: a result is off by half a step of its type, and by what its own sum of n products in
# float may be off, (n + 2) * 2^-24 of the magnitudes (norms and their gradients: 160, as derived beside their own tests).
@pytest.mark.gpu
@pytest.mark.parametrize("dt,act,context", [("bf16", "silu", True), ("bf16", "relu", False), ("f16", "relu", True), ("f16", "silu", False)])
def test_every_step_of_a_block(dt, act, context):
    mlp, d, ref, on1, on2 = setup(dt, act, M=70, d=192, f=320, context=context, training=True)
    M, width, hidden, U = 70, 192, 320, 2.0 ** -24
    values = {k: d[k] for k in ("gate", "post_weight", "pre_weight")}
    H_out, n = torch.empty_like(d["H"]), torch.empty_like(d["H"])
    mlp.forward(d["N"], d["H"], H_out, n, pre_bias=d["pre_bias"], **values)
    r = {k: v.detach() for k, v in ref.items()}
    half, tiny = torch.finfo(d["N"].dtype).eps / 2, torch.finfo(d["N"].dtype).smallest_normal * torch.finfo(d["N"].dtype).eps

    def of(t):
        return t.double().cpu()

    def step(what, got, want, mag, roundings=1):
        steps = 0.0 if got.dtype == torch.float32 else half * roundings * (1 + half)
        bound = steps * want.abs() + mag * U * (1 + 2 * half) + tiny
        err = (of(got) - want).abs()
        assert bool((err <= bound).all()), (what, float((err / bound).max()))
    W1, W2 = r["W1"] * on1, r["W2"] * on2
    # forward; an activation has a slope of 1.13 at most, and errs by 16 roundings of 1 + |z|
    z, mag = r["N"] @ W1 + r["b1"], (width + 2) * (r["N"].abs() @ W1.abs() + r["b1"].abs())
    step("a", mlp.a, torch.relu(z) if act == "relu" else z * torch.sigmoid(z), 1.13 * mag + 16 * (1 + z.abs()))
    if act != "relu":
        step("preact", mlp.preact, z, mag)
    a = of(mlp.a)
    step("y", mlp.y, a @ W2 + r["b2"], (hidden + 2) * (a.abs() @ W2.abs() + r["b2"].abs()))
    y = of(mlp.y)
    zy, mzy, ry = rows_standard(y, "rms")
    h, mh = 0.9 * r["H"] + r["gate"] * zy * r["post_weight"], 0.9 * r["H"].abs() + (r["gate"] * r["post_weight"]).abs() * mzy
    step("H_out", H_out, h, 160 * mh)
    zh, mzh, rh = rows_standard(h, "layer")
    extra = mh * rh + mh.mean(1, keepdim=True) * rh + zh.abs() * ((zh.abs() * mh).mean(1, keepdim=True) * rh)
    step("n", n, zh * r["pre_weight"] + r["pre_bias"], 160 * ((mzh + extra) * r["pre_weight"].abs() + r["pre_bias"].abs()))
    # backward
    g = torch.Generator().manual_seed(8)
    up_n, up_h = (torch.randn(M, width, generator=g).to(T[dt][1]) for _ in range(2))
    out = {"grad_N": torch.empty_like(d["N"]), "grad_H": torch.empty_like(d["H"]), **{"grad_" + k: torch.full(d[k].shape, float("nan"), device="cuda") for k in ("W1", "W2", "b1", "b2")}}
    mlp.backward(d["N"], H_out, grad_normed=up_n.cuda(), grad_H_out=up_h.cuda(), **values, **out)
    x, mx, rx = rows_standard(of(H_out), "layer")
    u, dh = of(up_n) * r["pre_weight"], of(up_h)
    dh, mdh = (dh + rx * (u - x * (u * x).mean(1, keepdim=True) - u.mean(1, keepdim=True)),
               dh.abs() + rx * (u.abs() + mx * (u.abs() * mx).mean(1, keepdim=True) + u.abs().mean(1, keepdim=True)))
    step("grad_H", out["grad_H"], 0.9 * dh, 160 * 0.9 * mdh)
    u, mu = dh * r["gate"] * r["post_weight"], mdh * (r["gate"] * r["post_weight"]).abs()
    step("grad_y", mlp.grad_y, ry * (u - zy * (u * zy).mean(1, keepdim=True)), 160 * ry * (mu + mzy * (mu * mzy).mean(1, keepdim=True)))
    dy = of(mlp.grad_y)
    step("grad_b2", out["grad_b2"], dy.sum(0), M * dy.abs().sum(0))
    step("grad_W2", out["grad_W2"], a.t() @ dy * on2, (M + 2) * (a.abs().t() @ dy.abs()) * on2)
    at = of(mlp.preact)
    slope = (at > 0).double() if act == "relu" else torch.sigmoid(at) * (1 + at * torch.sigmoid(-at))
    da, mda = dy @ W2.t(), (width + 2) * (dy.abs() @ W2.abs().t())
    step("grad_z", mlp.grad_a, da * slope, (mda + 16 * da.abs()) * (1.13 if act != "relu" else 1.0), roundings=2)   # (the product's, and behind the slope)
    dz = of(mlp.grad_a)
    step("grad_b1", out["grad_b1"], dz.sum(0), (M + half / U * (1 + 2 * half)) * dz.abs().sum(0))              # (summed before it is rounded)
    step("grad_W1", out["grad_W1"], r["N"].t() @ dz * on1, (M + 2) * (r["N"].abs().t() @ dz.abs()) * on1)
    step("grad_N", out["grad_N"], dz @ W1.t(), (hidden + 2) * (dz.abs() @ W1.abs().t()))
