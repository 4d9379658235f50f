"""The norms around a block, their gradients and the gradient through the epilogue, against the formulas in 64 bits on the host.

Bounds.  A value that is written to a type is off by half a step of it, eps / 2 of the value.  Before that it is float arithmetic: every
intermediate is off by at most S roundings of 2^-24, relative to the sum of the magnitudes of its terms, which the reference works out
next to the value (`mag`).  S: a sum over a row has at most 32 terms in a lane, 6 steps over the lanes and 16 over the waves (54), one over
rows at most 4 in a workgroup, 32 in a wave of the second launch and 16 waves for the sizes here (52); deviations and products add
fewer than 20.  A gradient goes through two such sums, one after the other: S = 160."""
import math

import pytest
import torch

import paper_2402_14118_amd as mm

T = {"f32": (mm.MMM_F32, torch.float32), "bf16": (mm.MMM_BF16, torch.bfloat16), "f16": (mm.MMM_F16, torch.float16)}
KINDS = {"none": mm.MMM_NORM_NONE, "rms": mm.MMM_NORM_RMS, "layer": mm.MMM_NORM_LAYER}
GATES = {"none": mm.MMM_GATE_NONE, "row": mm.MMM_GATE_ROW, "col": mm.MMM_GATE_COL, "full": mm.MMM_GATE_FULL}
S, U, EPS = 160, 2.0 ** -24, 1e-5


def check(got, want, mag, what):
    step = torch.finfo(got.dtype).eps / 2
    err = (got.double().cpu() - want).abs()
    bound = step * want.abs() + S * U * mag * (1 + step) + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    assert bool((err <= bound).all()), f"{what}: {int((~(err <= bound)).sum())} of {err.numel()} beyond the bound, by up to {float((err / bound).nan_to_num(9e9).max()):.3g}"


def standard(x, kind):
    """(x^, magnitude of its terms, 1 / deviation)"""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    am = x.abs().mean(1, keepdim=True) if kind == "layer" else 0.0
    r = 1 / ((x - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt()
    return (x - mean) * r, (x.abs() + am) * r, r


class Case:
    """Operands of a call on the device, in rows of `pad` elements more, and in 64 bits on the host."""

    def __init__(self, M, N, dt, stream, ytype, post, pre, gate, pad, affine, seed=0, block=True):
        self.__dict__.update(locals())
        g = torch.Generator().manual_seed(1000 * M + N + seed)
        self.dev, self.ref = {}, {}

        def make(name, shape, t, mean, std):
            v = (torch.randn(shape, generator=g) * std + mean).to(T[t][1])
            self.ref[name] = v.double()
            if len(shape) == 2:
                buf = torch.full((shape[0], shape[1] + pad), float("nan"), dtype=v.dtype)
                buf[:, : shape[1]] = v
                self.dev[name] = buf.cuda()[:, : shape[1]]
            else:
                buf = torch.full((shape[0] + 1,), float("nan"), dtype=v.dtype)   # (an odd start, where there is padding)
                buf[1 if pad else 0:][: shape[0]] = v
                self.dev[name] = buf.cuda()[1 if pad else 0:][: shape[0]]
        make("H", (M, N), stream, 0.3, 1.0)
        if block:
            make("Y", (M, N), ytype, -0.2, 2.0)
            if gate != "none":
                make("gate", {"row": (M,), "col": (N,), "full": (M, N)}[gate], dt, 0.2, 0.5)
        for at, on in (("post", post != "none"), ("pre", pre != "none")):
            if on and affine != "none":
                make(at + "_weight", (N,), dt, 1.0, 0.2)
                if affine == "both":
                    make(at + "_bias", (N,), dt, 0.0, 0.3)
        make("dn", (M, N), dt, 0.0, 1.0)
        make("dH_out", (M, N), stream, 0.0, 1.0)
        self.norm = mm.BlockNorm(M, N, T[dt][0], KINDS[post], KINDS[pre], GATES[gate] if block else 0, alpha=0.75, eps=EPS, dtype_h=T[stream][0],
                                 dtype_y=T[ytype][0], training=True)

    def out(self, shape, t):
        """Room for an output, whose padding has to stay as it is."""
        if len(shape) == 1:
            return torch.full(shape, float("nan"), device="cuda", dtype=T[t][1])
        return torch.full((shape[0], shape[1] + self.pad), 77.0, device="cuda", dtype=T[t][1])[:, : shape[1]]

    def untouched(self, t):
        whole = torch.as_strided(t, (t.shape[0], t.stride(0)), (t.stride(0), 1)) if t.dim() == 2 and t.shape[0] > 1 else t
        if t.dim() == 2 and t.shape[0] > 1 and self.pad:
            assert bool((whole[:-1, t.shape[1]:] == 77.0).all())

    def get(self, name):
        return self.ref.get(name)

    def spread(self):
        g = self.get("gate")
        return torch.ones(1, 1, dtype=torch.float64) if g is None else g[:, None] if self.gate == "row" else g

    def block_out(self):
        """v = norm(y) w + b: (value, magnitude, x^, its magnitude, r)"""
        y = self.ref["Y"]
        z, mz, r = standard(y, self.post) if self.post != "none" else (y, y.abs(), None)
        w = self.ref.get("post_weight", torch.ones(()).double())
        b = self.ref.get("post_bias", torch.zeros(()).double())
        return z * w + b, mz * w.abs() + b.abs(), z, mz, r

    def forward(self):
        h, mh = self.ref["H"], self.ref["H"].abs()
        if self.block:
            v, mv = self.block_out()[:2]
            h, mh = 0.75 * h + self.spread() * v, 0.75 * mh + self.spread().abs() * mv
        n = mn = None
        if self.pre != "none":
            w, b = self.ref.get("pre_weight", torch.ones(()).double()), self.ref.get("pre_bias", torch.zeros(()).double())
            z, mz, r = standard(h, self.pre)
            # an error of h' (its magnitude) goes through the deviation as well
            extra = mh * r + (mh.mean(1, keepdim=True) * r if self.pre == "layer" else 0.0) + z.abs() * ((z.abs() * mh).mean(1, keepdim=True) * r)
            n, mn = z * w + b, (mz + extra) * w.abs() + b.abs()
        return h, mh, n, mn

    def backward(self):
        out = {}
        d = self.ref["dH_out"]
        md = d.abs()
        if self.pre != "none":
            z, mz, r = standard(self.ref["H"], self.pre)
            dn = self.ref["dn"]
            u = dn * self.ref.get("pre_weight", torch.ones(()).double())
            out["grad_pre_weight"], out["grad_pre_bias"] = ((dn * z).sum(0), (dn.abs() * mz).sum(0)), (dn.sum(0), dn.abs().sum(0))
            lay = 1.0 if self.pre == "layer" else 0.0
            d = d + r * (u - z * (u * z).mean(1, keepdim=True) - lay * u.mean(1, keepdim=True))
            md = md + r * (u.abs() + mz * (u.abs() * mz).mean(1, keepdim=True) + lay * u.abs().mean(1, keepdim=True))
        if not self.block:
            out["grad_H"] = (d, md)
            return out
        out["grad_H"] = (0.75 * d, 0.75 * md)
        v, mv, z, mz, r = self.block_out()
        g = self.spread()
        dg, mdg = d * v, md * mv
        if self.gate == "row":
            out["grad_gate"] = (dg.sum(1), mdg.sum(1))
        elif self.gate == "col":
            out["grad_gate"] = (dg.sum(0), mdg.sum(0))
        elif self.gate == "full":
            out["grad_gate"] = (dg, mdg)
        dv, mdv = d * g, md * g.abs()
        if self.post == "none":
            out["grad_Y"] = (dv, mdv)
            return out
        out["grad_post_weight"], out["grad_post_bias"] = ((dv * z).sum(0), (mdv * mz).sum(0)), (dv.sum(0), mdv.sum(0))
        w = self.ref.get("post_weight", torch.ones(()).double())
        u, mu = dv * w, mdv * w.abs()
        lay = 1.0 if self.post == "layer" else 0.0
        out["grad_Y"] = (r * (u - z * (u * z).mean(1, keepdim=True) - lay * u.mean(1, keepdim=True)),
                         r * (mu + mz * (mu * mz).mean(1, keepdim=True) + lay * mu.mean(1, keepdim=True)))
        return out

    def run_forward(self):
        h_out = self.out((self.M, self.N), self.stream) if self.block else None
        n = self.out((self.M, self.N), self.dt) if self.pre != "none" else None
        d = self.dev
        self.norm.forward(d["H"], normed=n, H_out=h_out, **{k: d[k] for k in ("Y", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias") if k in d})
        return h_out, n

    def run_backward(self, want):
        shape = {"grad_H": ((self.M, self.N), self.stream), "grad_Y": ((self.M, self.N), self.ytype),
                 "grad_gate": {"row": ((self.M,), "f32"), "col": ((self.N,), "f32"), "full": ((self.M, self.N), self.dt)}.get(self.gate)}
        outs = {k: self.out(*shape.get(k, ((self.N,), "f32"))) for k in want}
        d, on = self.dev, self.pre != "none"
        self.norm.backward(H_out=d["H"] if on else None, grad_normed=d["dn"] if on else None, grad_H_out=d["dH_out"],
                           **{k: d[k] for k in ("Y", "gate", "post_weight", "post_bias", "pre_weight") if k in d}, **outs)
        return outs


# sizes: one element, below and across a piece of eight, across waves, across one piece per lane, odd, the widest
CASES = [
    (1, 1, "f32", "f32", "f32", "rms", "layer", "row", 0, "both"),
    (3, 7, "bf16", "bf16", "bf16", "layer", "rms", "col", 3, "both"),
    (5, 65, "f16", "f32", "f16", "rms", "rms", "full", 1, "weight"),
    (129, 513, "bf16", "f32", "f32", "layer", "layer", "row", 7, "both"),
    (777, 1992, "f32", "f32", "f32", "layer", "layer", "row", 0, "both"),
    (64, 1000, "f16", "f16", "f32", "none", "rms", "full", 0, "weight"),
    (17, 4096, "bf16", "bf16", "bf16", "rms", "none", "col", 8, "weight"),
    (2, 8200, "bf16", "bf16", "bf16", "rms", "rms", "none", 0, "none"),
    (3, 16391, "f32", "f32", "f32", "layer", "rms", "col", 1, "both"),
    (2, 32768, "f16", "f32", "f16", "layer", "layer", "col", 0, "both"),
    (9, 33, "f32", "f32", "f32", "none", "none", "row", 2, "none"),
    (1500, 40, "bf16", "bf16", "bf16", "none", "none", "row", 0, "none"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("args", CASES, ids=lambda a: "-".join(map(str, a)))
def test_both_directions(args):
    c = Case(*args)
    h, mh, n, mn = c.forward()
    got_h, got_n = c.run_forward()
    check(got_h, h, mh, "H_out")
    c.untouched(got_h)
    if n is not None:
        check(got_n, n, mn, "normed")
        c.untouched(got_n)
    want = c.backward()
    got = c.run_backward(want)
    again = c.run_backward(want)
    for k, (value, mag) in want.items():
        check(got[k], value, mag, k)
        assert torch.equal(got[k], again[k]), k   # no sum whose order changes
        if got[k].dim() == 2:
            c.untouched(got[k])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("M,N", [(1, 4096), (130, 100)])
def test_no_block(kind, M, N):
    """A norm alone, in front of a first block."""
    c = Case(M, N, "bf16", "bf16", "bf16", "none", kind, "none", 0, "both", block=False)
    _, n = c.run_forward()
    check(n, *c.forward()[2:], "normed")
    want = c.backward()
    got = c.run_backward(want)
    for k, (value, mag) in want.items():
        check(got[k], value, mag, k)


@pytest.mark.gpu
def test_in_place():
    """The residual stream and its gradient may be written where they were."""
    c = Case(33, 640, "bf16", "f32", "bf16", "rms", "rms", "col", 0, "weight")
    h_out, n = c.run_forward()
    d = dict(c.dev)
    stream, n2 = d["H"].clone(), torch.empty_like(n)
    c.norm.forward(stream, normed=n2, H_out=stream, Y=d["Y"], gate=d["gate"], post_weight=d["post_weight"], pre_weight=d["pre_weight"])
    assert torch.equal(stream, h_out) and torch.equal(n2, n)
    want = c.run_backward(["grad_H", "grad_Y"])
    grad, dy = d["dH_out"].clone(), torch.empty_like(d["Y"])
    c.norm.backward(H_out=d["H"], grad_normed=d["dn"], grad_H_out=grad, grad_H=grad, Y=d["Y"], gate=d["gate"], grad_Y=dy,
                    post_weight=d["post_weight"], pre_weight=d["pre_weight"])
    assert torch.equal(grad, want["grad_H"]) and torch.equal(dy, want["grad_Y"])


@pytest.mark.gpu
def test_rows_without_contrast_and_rows_that_are_not_finite():
    """Zero and constant rows are held by eps; a row that is not finite is that row's alone."""
    M, N = 6, 200
    H = torch.randn(M, N, device="cuda")
    H[1], H[2], H[3, 7], H[4, 9] = 0.0, 5.0, float("inf"), float("nan")
    n = torch.empty_like(H)
    for kind in (mm.MMM_NORM_RMS, mm.MMM_NORM_LAYER):
        mm.BlockNorm(M, N, mm.MMM_F32, pre=kind, eps=EPS).forward(H, normed=n)
        x = H.double().cpu()
        for row in (0, 1, 2, 5):
            z, mz, _ = standard(x[row: row + 1], "rms" if kind == mm.MMM_NORM_RMS else "layer")
            check(n[row: row + 1], z, mz, f"row {row}")
        assert bool(n[4].isnan().all()) and bool(n[3, 7].isnan())


@pytest.mark.gpu
def test_gradients_against_differences():
    """(f(p + e) - f(p - e)) / 2 e of f = sum(d_n n + d_h' h') in 64 bits, along random directions of every input.  The difference errs by e^2 / 6
    of the third derivative; the inputs are of order one, and e = 2^-10 of them leaves less than 1e-4 of the sum of magnitudes."""
    c = Case(7, 48, "f32", "f32", "f32", "layer", "rms", "col", 0, "both")
    h_out, _ = c.run_forward()
    # the backward call is at the stream behind the block
    d = c.dev
    outs = {"grad_H": torch.empty_like(d["H"]), "grad_Y": torch.empty_like(d["Y"]), **{k: torch.empty(48, device="cuda") for k in
            ("grad_gate", "grad_post_weight", "grad_post_bias", "grad_pre_weight", "grad_pre_bias")}}
    c.norm.backward(H_out=h_out, grad_normed=d["dn"], grad_H_out=d["dH_out"], Y=d["Y"], gate=d["gate"], post_weight=d["post_weight"],
                    post_bias=d["post_bias"], pre_weight=d["pre_weight"], **outs)

    def f():
        h, _, n, _ = c.forward()
        return float((c.ref["dn"] * n).sum() + (c.ref["dH_out"] * h).sum())
    g = torch.Generator().manual_seed(5)
    for name in ("H", "Y", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias"):
        at, e = c.ref[name], 2.0 ** -10
        way = torch.randn(at.shape, generator=g).double()
        c.ref[name] = at + e * way
        up = f()
        c.ref[name] = at - e * way
        down = f()
        c.ref[name] = at
        terms = outs["grad_" + name].double().cpu() * way
        assert abs((up - down) / (2 * e) - float(terms.sum())) <= 1e-4 * float(terms.abs().sum()), name


@pytest.mark.gpu
def test_another_stream_and_a_replayed_graph():
    c = Case(64, 1000, "bf16", "bf16", "bf16", "rms", "layer", "col", 0, "both")
    want_f, keys = c.run_forward(), list(c.backward())
    want_b = c.run_backward(keys)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        f, b = c.run_forward(), c.run_backward(keys)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(f, want_f)) and all(torch.equal(b[k], want_b[k]) for k in keys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f, b = c.run_forward(), c.run_backward(keys)
    for _ in range(3):
        for t in (*f, *b.values()):
            t.fill_(0.0)
        c.run_backward(keys)   # the program's own work between replays, on the same workspace and stream
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(f, want_f)) and all(torch.equal(b[k], want_b[k]) for k in keys)


# ---- the gradient through the epilogue

ACTS = {"none": mm.MMM_ACT_NONE, "relu": mm.MMM_ACT_RELU, "gelu": mm.MMM_ACT_GELU, "gelu_tanh": mm.MMM_ACT_GELU_TANH, "silu": mm.MMM_ACT_SILU}


def slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(8 / math.pi)
        p = torch.sigmoid(a * (z + 0.044715 * z ** 3))
        return p + z * p * torch.sigmoid(-a * (z + 0.044715 * z ** 3)) * a * (1 + 0.134145 * z * z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * torch.sigmoid(-z)
    return torch.ones_like(z)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,dt,out,pad", [(1, 8, "f32", "f32", 0), (5, 13, "bf16", "bf16", 3), (777, 1992, "f16", "f32", 0), (300, 1031, "bf16", "f32", 1),
                                           (2049, 520, "f16", "f16", 8)])
def test_epilogue_backward(act, M, N, dt, out, pad):
    """The slope of a smooth activation is off by the error of its exponential's argument, 2^-24 (1 + z^2) of terms of at most 1 + |z|: |z| < 8
    here, so less than 8 * 16 * 65 / 2 roundings where it is largest and S of the magnitude below."""
    g = torch.Generator().manual_seed(M + N)

    def room(v, t):
        buf = torch.full((M, N + pad), 77.0, dtype=T[t][1])
        buf[:, :N] = v.to(T[t][1])
        return buf.cuda()[:, :N]
    dC, Z = room(torch.randn(M, N, generator=g), out), room(torch.randn(M, N, generator=g) * 1.5, out)
    dZ = room(torch.zeros(M, N), dt)
    dbias = torch.empty(N, device="cuda")
    need = mm.mmm_epilogue_backward_workspace_bytes(M, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(dZ=dZ, dbias=dbias, dC=dC):
        mm.mmm_epilogue_backward(M, N, T[dt][0], T[out][0], ACTS[act], dC, N + pad, Z if act != "none" else None, N + pad, dZ, N + pad, dbias, ws, need)
    call()
    z, d = Z.double().cpu(), dC.double().cpu()
    want, mag = d * slope(z, act), d.abs() * (1 + z.abs()) * (1 + z * z / 8)
    check(dZ, want, mag, "dZ")
    check(dbias, want.sum(0), mag.sum(0), "dbias")
    if M > 1 and pad:
        assert bool((torch.as_strided(dZ, (M - 1, N + pad), (N + pad, 1))[:, N:] == 77.0).all())
    alone, sums = torch.full((M, N + pad), 77.0, device="cuda", dtype=T[dt][1])[:, :N], torch.empty_like(dbias)
    call(dZ=alone, dbias=None)
    call(dZ=None, dbias=sums)
    assert torch.equal(alone, dZ) and torch.equal(sums, dbias)
    if dt == out:   # in place
        own = dC.clone(memory_format=torch.preserve_format)
        if own.stride(0) == N + pad:
            mm.mmm_epilogue_backward(M, N, T[dt][0], T[out][0], ACTS[act], own, N + pad, Z if act != "none" else None, N + pad, own, N + pad, None, None, 0)
            assert torch.equal(own, dZ)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
def test_slopes_at_the_ends(act):
    """Large, infinite and zero arguments: the limits, and the definition at 0; NaN stays NaN."""
    Z = torch.tensor([[0.0, -0.0, 1e4, -1e4, 3e38, -3e38, float("inf"), -float("inf"), 20.0, -20.0, 1e-30, float("nan")]], device="cuda")
    dC, dZ, n = torch.full_like(Z, 2.0), torch.empty_like(Z), Z.shape[1]
    mm.mmm_epilogue_backward(1, n, mm.MMM_F32, mm.MMM_F32, ACTS[act], dC, n, Z, n, dZ, n)
    got = dZ.cpu()[0].tolist()
    at0 = {"none": 2.0, "relu": 0.0}.get(act, 1.0)
    low = 2.0 if act == "none" else 0.0
    assert got[0] == at0 and got[1] == at0
    assert got[2] == got[4] == got[6] == 2.0 and got[3] == got[5] == got[7] == low
    assert abs(got[8] - 2.0) < 1e-6 and abs(got[9] - low) < 1e-6
    assert act == "none" or math.isnan(got[11])


@pytest.mark.gpu
def test_more_elements_than_32_bits_count():
    """The last rows of matrices of more than 2^32 elements come out as those of a matrix of their own; sums of whole numbers are exact."""
    M, N, tail = 131100, 32768, 64
    g = torch.Generator().manual_seed(2)
    ends = [torch.randint(-3, 4, (tail, N), generator=g).bfloat16().cuda() for _ in range(3)]
    whole = [torch.ones(M, N, dtype=torch.bfloat16, device="cuda") for _ in ends]
    for w, e in zip(whole, ends):
        w[-tail:] = e
    (H, Y, D), out, results = whole, torch.empty_like(whole[0]), []
    for rows, (h, y, d, to) in ((tail, (*ends, torch.empty_like(ends[0]))), (M, (H, Y, D, out))):
        norm = mm.BlockNorm(rows, N, mm.MMM_BF16, post=mm.MMM_NORM_RMS, training=True)
        norm.forward(h, normed=to, H_out=h, Y=y)          # (in place)
        parts = [h[-tail:].clone(), to[-tail:].clone()]
        norm.backward(H_out=h, grad_normed=d, grad_H=to, Y=y)
        parts.append(to[-tail:].clone())
        dbias = torch.empty(N, device="cuda")
        ws = torch.empty(mm.mmm_epilogue_backward_workspace_bytes(rows, N), dtype=torch.uint8, device="cuda")
        mm.binding.mmm_epilogue_backward(rows, N, mm.MMM_BF16, mm.MMM_BF16, mm.MMM_ACT_RELU, y, N, y, N, to, N, dbias, ws, ws.numel())
        assert torch.equal(dbias, ends[1].float().clamp(min=0).sum(0) + (rows - tail))
        results.append(parts + [to[-tail:].clone()])
    assert all(torch.equal(a, b) for a, b in zip(*results))


# several rows side by side in a workgroup: fewer rows than that, some left over, more than one turn
@pytest.mark.gpu
@pytest.mark.parametrize("args", [(1, 512, "bf16", "bf16", "bf16", "rms", "rms", "col", 0, "weight"), (5, 8, "f32", "f32", "f32", "layer", "rms", "full", 1, "both"),
                                  (13, 1024, "f16", "f32", "f16", "rms", "layer", "row", 3, "both"), (3, 2048, "bf16", "f32", "f32", "layer", "layer", "none", 0, "weight"),
                                  (2500, 72, "bf16", "bf16", "bf16", "rms", "rms", "col", 0, "weight"), (1541, 640, "f32", "f32", "f32", "rms", "rms", "full", 0, "weight"),
                                  (1031, 1032, "f16", "f16", "f32", "layer", "none", "row", 8, "both")], ids=lambda a: "-".join(map(str, a)))
def test_rows_side_by_side(args):
    c = Case(*args)
    want = c.backward()
    got = c.run_backward(list(want))
    for k, (w, mag) in want.items():
        check(got[k], w, mag, k)
        c.untouched(got[k])
    again = c.run_backward(list(want))
    assert all(torch.equal(got[k], again[k]) for k in want)
