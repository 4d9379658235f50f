"""The operators around the masked product as timed and compared cases.

A case names one operator, its sizes, types and masks:

  "product"          C = act(M(X) x N(Y) + bias) + residual
  "product_grad"     dX = M .* (dC x N(Y)^T), dY = N .* (M(X)^T x dC): the gradients under the maps as built
  "activation_grad"  dZ = dC .* act'(Z), dbias = its column sums
  "norm"             v = norm(y), h' = alpha h + gate v, n = norm(h'): behind a block, and in front of the next one
  "norm_grad"        the gradients of all of its inputs

`own` false: the plain form, elementary torch operations in 32 bits (64 for doubles), rounded once.  `own` true: the engine's calls.

Use of the product: "step" (both operands are new), "cached" (Y is a weight matrix whose map was built once), "fused" (the
same, few rows: the mask of X is evaluated inside the multiplication).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f64": torch.float64}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "f64": 8}


def _relu_share(mu):
    """Share of N(mu, 1) that is positive."""
    return 0.5 * math.erfc(-mu / math.sqrt(2.0))


def _product(dtype, use, M, K, N, bw, mu, p_b, p_rows, act, bias, residual, preact, **name):
    """mu: X ~ N(mu, 1) under the predicate x > 0; None: X ~ N(0, 1), every element counts."""
    return dict(name, op="product", dtype=dtype, use=use, M=M, K=K, N=N, bw=bw, relu=mu is not None, mu=mu or 0.0, p_b=p_b, p_rows=p_rows,
                act=act, bias=bias, residual=residual, preact=preact)


def _product_grad(dtype, M, K, N, bw, mu, p_b, p_rows, **name):
    return dict(name, op="product_grad", dtype=dtype, M=M, K=K, N=N, bw=bw, relu=mu is not None, mu=mu or 0.0, p_b=p_b, p_rows=p_rows)


def _activation_grad(dtype, M, N, act, bias, **name):
    return dict(name, op="activation_grad", dtype=dtype, M=M, N=N, act=act, bias=bias)


def _norm(op, dtype, stream, M, N, kind, post, pre, gate, alpha, affine, **name):
    """stream: type of the residual stream h, h'; affine: "weight" or "both" (weight and bias)."""
    return dict(name, op=op, dtype=dtype, stream=stream, M=M, N=N, kind=kind, post=post, pre=pre, gate=gate, alpha=alpha, affine=affine)


def listed():
    return [
        # decode of a few tokens: down-projection of ReLU activations, bias and residual in the same launch
        _product("bf16", "fused", 4, 16384, 4096, 16, -1.65, 0.1, 0.0, "none", True, True, False, name="decode_4_down_bf16"),
        # prefill: the up-projection of dense rows whose ReLU makes the sparsity, weights cached, output in 16 bits
        _product("bf16", "cached", 2048, 4096, 16384, 32, None, 1.0, 0.0, "relu", True, False, False, name="up_2048_bf16"),
        # the down-projection behind it, neurons selected by context, single precision
        _product("f32", "step", 2048, 16384, 4096, 32, -1.3, 0.5, 0.1, "none", True, True, False, name="down_2048_f32"),
        # sizes that divide nothing, half precision, narrow blocks, a smooth activation whose argument is kept for training
        _product("f16", "step", 777, 3001, 1992, 8, -1.0, 0.15, 0.0, "gelu", True, False, True, name="ragged_777_f16"),
        # training of the down-projection: ReLU activations, dense 16-bit weights
        _product_grad("bf16", 2048, 16384, 4096, 32, -1.3, 1.0, 0.0, name="grad_down_2048_bf16"),
        # the same of a ragged problem in single precision, rows by context
        _product_grad("f32", 777, 3001, 1992, 8, -1.0, 0.5, 0.25, name="grad_ragged_777_f32"),
        # the gradient through the up-projection's ReLU and bias
        _activation_grad("bf16", 2048, 16384, "relu", True, name="grad_relu_2048_bf16"),
        # a smooth activation on odd sizes
        _activation_grad("f16", 777, 1992, "gelu", True, name="grad_gelu_777_f16"),
        # decode: behind a block and in front of the next, a few rows
        _norm("norm", "bf16", "bf16", 4, 4096, "rms", True, True, "col", 1.0, "weight", name="norm_4_bf16"),
        # prefill or training: the same over 2048 tokens
        _norm("norm", "bf16", "bf16", 2048, 4096, "rms", True, True, "col", 1.0, "weight", name="norm_2048_bf16"),
        # its gradients
        _norm("norm_grad", "bf16", "bf16", 2048, 4096, "rms", True, True, "col", 1.0, "weight", name="grad_norm_2048_bf16"),
        # mean and variance, a gate per token, a scaled residual, odd sizes, single precision
        _norm("norm_grad", "f32", "f32", 777, 1992, "layer", True, True, "row", 0.8, "both", name="grad_norm_777_f32"),
    ]


def _size(rng, lo, hi, unit=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(unit, min(hi, int(round(v / unit)) * unit))


def draw(rng):
    op = rng.choice(["product", "product", "product_grad", "activation_grad", "norm", "norm_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "activation_grad":
        return _activation_grad(dtype, _size(rng, 1, 2048), _size(rng, 64, 16384), rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), rng.random() < 0.7)
    if op in ("norm", "norm_grad"):
        post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        # with a norm in front only there may be no block before it
        gate = rng.choice(["none", "row", "col", "full"])
        stream = rng.choice([dtype, "f32"])
        return _norm(op, dtype, stream, _size(rng, 1, 2048), _size(rng, 64, 4096), rng.choice(["rms", "layer"]), post, pre, gate,
                     rng.choice([1.0, 1.0, round(rng.uniform(0.5, 1.5), 2)]), rng.choice(["weight", "both"]))
    while True:
        bw = rng.choice([8, 16, 32])
        mu = rng.choice([None, round(rng.uniform(-1.65, -0.5), 2)])
        p_rows = rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.3), 2)])
        p_b = round(math.exp(rng.uniform(math.log(0.1), 0.0)), 2)
        K, N = _size(rng, 200, 16384), _size(rng, 200, 16384, bw)
        if op == "product_grad":
            c = _product_grad(dtype, _size(rng, 16, 2048), K, N, bw, mu, p_b, p_rows)
        else:
            use = rng.choice(["step", "cached", "cached", "fused"])
            if rng.random() < 0.1:
                dtype, p_rows = "f64", 0.0
            M = _size(rng, 1, 16) if use == "fused" else _size(rng, 1, 2048)
            if use == "fused":
                p_rows = 0.0
            c = _product(dtype, use, M, K, N, bw, mu, p_b, p_rows, rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), rng.random() < 0.8,
                         rng.random() < 0.5, rng.random() < 0.3)
        # nothing above the listed ones (doubles, and vector units for few rows, cost more per product)
        most = {"f64": 2.0 ** 31, "f32": 2.0 ** 36}.get(dtype, 2.0 ** 37)
        if float(c["M"]) * K * N * p_b * (p_rows or 1.0) <= most and float(c["M"]) * K * N <= 2.0 ** 37 and (c["op"] != "product" or c["use"] != "fused" or p_b <= 0.2):
            return c


# ---- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, mean, std, dtype):
    wide = torch.float64 if dtype == torch.float64 else torch.float32
    return torch.randn(shape, generator=g, device="cuda", dtype=wide).mul_(std).add_(mean).to(dtype)


def _words(flags):
    """Boolean [rows, cols] to the engine's bitmaps: 64-bit words, lowest bit first, rows padded to whole words."""
    rows, cols = flags.shape
    words = (cols + 63) // 64
    padded = torch.zeros((rows, words * 64), dtype=torch.uint8, device=flags.device)
    padded[:, :cols] = flags
    weights = torch.tensor([1, 2, 4, 8, 16, 32, 64, 128], dtype=torch.uint8, device=flags.device)
    by = (padded.view(rows, words * 8, 8) * weights).sum(dim=-1, dtype=torch.uint8)
    return by.view(torch.int64).contiguous()


def _inputs(case, seed):
    """The tensors a call is made with, from the seed alone."""
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    s = {}
    if case["op"] in ("product", "product_grad"):
        M, K, N, bw = case["M"], case["K"], case["N"], case["bw"]
        s["X"] = _normal(g, (M, K), case["mu"], 1.0, dt)
        s["Y"] = _normal(g, (K, N), 0.0, 0.02, dt)
        s["keep_rows"] = torch.rand((1, K), generator=g, device="cuda") < case["p_rows"] if case["p_rows"] > 0 else None
        s["keep_blocks"] = torch.rand((K, N // bw), generator=g, device="cuda") < case["p_b"] if case["p_b"] < 1 else None
        if case["op"] == "product":
            s["bias"] = _normal(g, (N,), 0.0, 0.1, dt) if case["bias"] else None
            s["residual"] = _normal(g, (M, N), 0.0, 1.0, dt) if case["residual"] else None
        else:
            s["dC"] = _normal(g, (M, N), 0.0, 1.0, dt)
    elif case["op"] == "activation_grad":
        M, N = case["M"], case["N"]
        s["dC"], s["Z"] = _normal(g, (M, N), 0.0, 1.0, dt), _normal(g, (M, N), -0.5, 1.0, dt)
    else:
        M, N, ds = case["M"], case["N"], DTYPES[case["stream"]]
        s["H"] = _normal(g, (M, N), 0.1, 1.0, ds)
        if case["post"]:
            s["Y"] = _normal(g, (M, N), 0.2, 0.7, dt)
            shape = {"none": None, "row": (M,), "col": (N,), "full": (M, N)}[case["gate"]]
            s["gate"] = _normal(g, shape, 0.3, 0.3, dt) if shape else None
            s["post_weight"] = _normal(g, (N,), 1.0, 0.1, dt)
            s["post_bias"] = _normal(g, (N,), 0.0, 0.1, dt) if case["affine"] == "both" else None
        if case["pre"]:
            s["pre_weight"] = _normal(g, (N,), 1.0, 0.1, dt)
            s["pre_bias"] = _normal(g, (N,), 0.0, 0.1, dt) if case["affine"] == "both" else None
        if case["op"] == "norm_grad":
            # H is then the stream behind the block, as the forward call left it
            if case["pre"]:
                s["dn"] = _normal(g, (M, N), 0.0, 1.0, dt)
            s["dH_out"] = _normal(g, (M, N), 0.0, 1.0, ds)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        if case["op"] in ("product", "product_grad"):
            # the weights as the masks leave them: laid out once where the weights stay
            if case["op"] == "product_grad" or case["use"] != "step":
                s["B"] = _kept(s["Y"], s["keep_rows"], s["keep_blocks"], case["bw"])
        return s
    import paper_2402_14118_amd as mm
    s["mm"] = mm
    code = {"f32": mm.MMM_F32, "bf16": mm.MMM_BF16, "f16": mm.MMM_F16, "f64": mm.MMM_F64}
    act = {"none": mm.MMM_ACT_NONE, "relu": mm.MMM_ACT_RELU, "gelu": mm.MMM_ACT_GELU, "gelu_tanh": mm.MMM_ACT_GELU_TANH, "silu": mm.MMM_ACT_SILU}
    dt = DTYPES[case["dtype"]]
    if case["op"] in ("product", "product_grad"):
        M, K, N = case["M"], case["K"], case["N"]
        rows, blocks = (None if s[k] is None else _words(s[k]) for k in ("keep_rows", "keep_blocks"))
        s["rows"], s["blocks"], s["pred"] = rows, blocks, mm.MMM_PRED_GT if case["relu"] else mm.MMM_PRED_NONZERO
        eng = s["eng"] = mm.MaskedMatmul(M, K, N, case["bw"], code[case["dtype"]])
        if case["op"] == "product" and case["use"] == "fused":
            eng.build_maps(None, s["Y"], keep_rows=rows, keep_blocks=blocks)
        else:
            # as a program does once per layer: the maps of its first inputs, and the engine's count of their densities
            eng.build_maps(s["X"], s["Y"], s["pred"], 0.0, None, rows, blocks)
            eng.stats()
        if case["op"] == "product":
            s["act"] = act[case["act"]]
            s["C"] = torch.empty((M, N), dtype=dt, device="cuda")
            s["preact"] = torch.empty((M, N), dtype=dt, device="cuda") if case["preact"] else None
        else:
            s["dX"] = torch.empty((M, K), dtype=dt, device="cuda")
            s["dY"] = torch.empty((K, N), dtype=torch.float32, device="cuda")
    elif case["op"] == "activation_grad":
        M, N = case["M"], case["N"]
        s["act"], s["code"] = act[case["act"]], code[case["dtype"]]
        s["dZ"] = torch.empty((M, N), dtype=dt, device="cuda")
        s["dbias"] = torch.empty((N,), dtype=torch.float32, device="cuda") if case["bias"] else None
        s["ws"] = torch.empty((mm.mmm_epilogue_backward_workspace_bytes(M, N),), dtype=torch.uint8, device="cuda")
    else:
        M, N, ds = case["M"], case["N"], DTYPES[case["stream"]]
        kind = mm.MMM_NORM_RMS if case["kind"] == "rms" else mm.MMM_NORM_LAYER
        gate = {"none": mm.MMM_GATE_NONE, "row": mm.MMM_GATE_ROW, "col": mm.MMM_GATE_COL, "full": mm.MMM_GATE_FULL}[case["gate"]] if case["post"] else mm.MMM_GATE_NONE
        s["norm"] = mm.BlockNorm(M, N, code[case["dtype"]], post=kind if case["post"] else mm.MMM_NORM_NONE, pre=kind if case["pre"] else mm.MMM_NORM_NONE,
                                 gate=gate, alpha=case["alpha"], eps=1e-5, dtype_h=code[case["stream"]], training=case["op"] == "norm_grad")

        def new(shape, dtype):
            return torch.empty(shape, dtype=dtype, device="cuda")
        if case["op"] == "norm":
            s["n"] = new((M, N), dt) if case["pre"] else None
            s["h_out"] = new((M, N), ds) if case["post"] else None
        else:
            s["dH"] = new((M, N), ds)
            both = case["affine"] == "both"
            if case["post"]:
                s["dY"] = new((M, N), dt)
                s["dgate"] = {"none": lambda: None, "row": lambda: new((M,), torch.float32), "col": lambda: new((N,), torch.float32),
                              "full": lambda: new((M, N), dt)}[case["gate"]]()
                s["dpost_weight"], s["dpost_bias"] = new((N,), torch.float32), new((N,), torch.float32) if both else None
            if case["pre"]:
                s["dpre_weight"], s["dpre_bias"] = new((N,), torch.float32), new((N,), torch.float32) if both else None
    return s


# ---- the plain form

def _kept(Y, keep_rows, keep_blocks, bw):
    """N(Y): the blocks that the masks leave on, zeros elsewhere."""
    if keep_rows is None and keep_blocks is None:
        return Y
    on = torch.ones_like(Y, dtype=torch.bool)
    if keep_blocks is not None:
        on = on & keep_blocks.repeat_interleave(bw, dim=1)
    if keep_rows is not None:
        on = on & keep_rows.view(-1, 1)
    return torch.where(on, Y, torch.zeros((), dtype=Y.dtype, device=Y.device))


def _blocks_on(B, bw):
    """Where a block of N(Y) holds anything, element by element."""
    return (B.view(B.shape[0], -1, bw) != 0).any(dim=2).repeat_interleave(bw, dim=1)


def _activated(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * z * z)
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    return torch.ones_like(z)


def _standard(x, kind):
    """(x standardised, 1 / its deviation), row by row."""
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + 1e-5)
    return x * r, r


def _standard_grad(d, xhat, r, kind):
    d_in = d - xhat * (d * xhat).mean(dim=1, keepdim=True)
    if kind == "layer":
        d_in = d_in - d.mean(dim=1, keepdim=True)
    return d_in * r


def _spread(gate, kind):
    return gate.view(-1, 1) if kind == "row" else gate


def _plain(s):
    case = s["case"]
    dt = DTYPES[case["dtype"]]
    wide = torch.float64 if case["dtype"] == "f64" else torch.float32

    def f(name):
        return s[name].to(wide)
    if case["op"] in ("product", "product_grad"):
        on = s["X"] > 0 if case["relu"] else s["X"] != 0
        A = torch.where(on, f("X"), torch.zeros((), dtype=wide, device="cuda"))
        kept = s["B"] if "B" in s else _kept(s["Y"], s["keep_rows"], s["keep_blocks"], case["bw"])
        B = kept.to(wide)
        if case["op"] == "product_grad":
            dC = f("dC")
            return [torch.where(on, dC @ B.t(), torch.zeros((), dtype=wide, device="cuda")).to(dt),
                    torch.where(_blocks_on(kept, case["bw"]), A.t() @ dC, torch.zeros((), dtype=wide, device="cuda"))]
        z = A @ B
        if s["bias"] is not None:
            z = z + f("bias")
        c = _activated(z, case["act"])
        if s["residual"] is not None:
            c = c + f("residual")
        return [c.to(dt)] + ([z.to(dt)] if case["preact"] else [])
    if case["op"] == "activation_grad":
        dZ = f("dC") * _slope(f("Z"), case["act"])
        return [dZ.to(dt)] + ([dZ.sum(dim=0)] if case["bias"] else [])
    kind, ds, gate = case["kind"], DTYPES[case["stream"]], case["gate"] if case["post"] else "none"
    h, out = f("H"), []
    if case["post"]:
        yhat, ry = _standard(f("Y"), kind)
        v = yhat * f("post_weight") + (f("post_bias") if s["post_bias"] is not None else 0.0)
        gated = v if gate == "none" else _spread(f("gate"), gate) * v
    if case["op"] == "norm":
        if case["post"]:
            h = case["alpha"] * h + gated
            out.append(h.to(ds))
        if case["pre"]:
            n = _standard(h, kind)[0] * f("pre_weight")
            out.append((n + f("pre_bias") if s["pre_bias"] is not None else n).to(dt))
        return out
    d = f("dH_out")
    if case["pre"]:
        xhat, r = _standard(h, kind)
        dn = f("dn")
        d = d + _standard_grad(dn * f("pre_weight"), xhat, r, kind)
        out.append((dn * xhat).sum(dim=0))
        if s["pre_bias"] is not None:
            out.append(dn.sum(dim=0))
    if not case["post"]:
        return [d.to(ds)] + out
    dv = d if gate == "none" else d * _spread(f("gate"), gate)
    out += [(dv * yhat).sum(dim=0)] + ([dv.sum(dim=0)] if s["post_bias"] is not None else [])
    if gate != "none":
        dg = d * v
        out.append(dg.sum(dim=1) if gate == "row" else dg.sum(dim=0) if gate == "col" else dg.to(dt))
    return [(case["alpha"] * d).to(ds)] + out + [_standard_grad(dv * f("post_weight"), yhat, ry, kind).to(dt)]


def run(state):
    s = state
    if not own:
        return _plain(s)
    case, mm = s["case"], s["mm"]
    if case["op"] == "product":
        eng = s["eng"]
        if case["use"] == "step":
            eng.build_maps(s["X"], s["Y"], s["pred"], 0.0, None, s["rows"], s["blocks"])
        elif case["use"] == "cached":
            eng.build_maps(s["X"], None, s["pred"], 0.0)
        eng.matmul_epilogue(s["X"], s["Y"], s["C"], bias=s["bias"], activation=s["act"], residual=s["residual"], preact=s["preact"],
                            pred=s["pred"] if case["use"] == "fused" else None)
        return [s["C"]] + ([s["preact"]] if case["preact"] else [])
    if case["op"] == "product_grad":
        # (the maps are those of the forward pass)
        s["eng"].matmul_backward(s["X"], s["Y"], s["dC"], dX=s["dX"], dY=s["dY"])
        return [s["dX"], s["dY"]]
    if case["op"] == "activation_grad":
        M, N = case["M"], case["N"]
        mm.mmm_epilogue_backward(M, N, s["code"], s["code"], s["act"], s["dC"], N, s["Z"], N, s["dZ"], N, s["dbias"], s["ws"], s["ws"].numel())
        return [s["dZ"]] + ([s["dbias"]] if case["bias"] else [])
    g = s.get
    if case["op"] == "norm":
        s["norm"].forward(s["H"], normed=s["n"], H_out=s["h_out"], Y=g("Y"), gate=g("gate"), post_weight=g("post_weight"), post_bias=g("post_bias"),
                          pre_weight=g("pre_weight"), pre_bias=g("pre_bias"))
        return [t for t in (s["h_out"], s["n"]) if t is not None]
    s["norm"].backward(H_out=s["H"], grad_normed=g("dn"), grad_H_out=s["dH_out"], grad_H=s["dH"], Y=g("Y"), gate=g("gate"), post_weight=g("post_weight"),
                       post_bias=g("post_bias"), pre_weight=g("pre_weight"), grad_Y=g("dY"), grad_gate=g("dgate"), grad_post_weight=g("dpost_weight"),
                       grad_post_bias=g("dpost_bias"), grad_pre_weight=g("dpre_weight"), grad_pre_bias=g("dpre_bias"))
    return [t for t in (s["dH"], g("dpre_weight"), g("dpre_bias"), g("dpost_weight"), g("dpost_bias"), g("dgate"), g("dY")) if t is not None]


def work(case):
    """Every input and output once; the products that both masks leave (the gradients: in each of the two)."""
    e, M, N = SIZES[case["dtype"]], case["M"], case["N"]
    if case["op"] in ("product", "product_grad"):
        K, bw = case["K"], case["bw"]
        share = case["p_b"] * (case["p_rows"] or 1.0)
        p_a = _relu_share(case["mu"]) if case["relu"] else 1.0
        nbytes = M * K * e + K * N * e * share + (K * (N // bw) / 8 if case["p_b"] < 1 else 0)
        flops = 2.0 * M * K * N * p_a * share
        if case["op"] == "product":
            return {"bytes": nbytes + M * N * e * (1 + case["residual"] + case["preact"]), "flops": flops}
        return {"bytes": nbytes + M * N * e + M * K * e + K * N * 4, "flops": 2 * flops}
    if case["op"] == "activation_grad":
        return {"bytes": M * N * e * 3 + (N * 4 if case["bias"] else 0), "flops": 4.0 * M * N}
    h = SIZES[case["stream"]]
    full = case["post"] and case["gate"] == "full"
    if case["op"] == "norm":
        per = h + (e + h if case["post"] else 0) + (e if case["pre"] else 0) + (e if full else 0)
        return {"bytes": M * N * per, "flops": 12.0 * M * N}
    per = 2 * h + (h + e if case["pre"] else 0) + (2 * e if case["post"] else 0) + (2 * e if full else 0)
    return {"bytes": M * N * per, "flops": 30.0 * M * N}


# ---- the definition in 64 bits

def exact(case, seed):
    s = {k: (v.double() if v is not None and v.is_floating_point() else v) for k, v in _inputs(case, seed).items()}
    if case["op"] in ("product", "product_grad"):
        A = s["X"].clamp(min=0.0) if case["relu"] else s["X"]
        weight = torch.ones((case["K"], case["N"] // case["bw"]), dtype=torch.float64, device="cuda")
        if s["keep_rows"] is not None:
            weight *= s["keep_rows"].reshape(-1, 1)
        if s["keep_blocks"] is not None:
            weight *= s["keep_blocks"]
        pieces = s["Y"].reshape(case["K"], -1, case["bw"]) * weight.unsqueeze(2)
        B = pieces.reshape(case["K"], case["N"])
        if case["op"] == "product_grad":
            occupied = (pieces.abs().amax(dim=2, keepdim=True) > 0).double().expand_as(pieces).reshape(B.shape)
            return [torch.mm(s["dC"], B.t().contiguous()) * (A != 0), torch.mm(A.t().contiguous(), s["dC"]) * occupied]
        z = torch.mm(A, B)
        if s["bias"] is not None:
            z += s["bias"]
        c = {"none": lambda: z, "relu": lambda: z.clamp(min=0.0), "gelu": lambda: z * 0.5 * torch.erfc(-z / math.sqrt(2.0)),
             "gelu_tanh": lambda: z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)), "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        if s["residual"] is not None:
            c = c + s["residual"]
        return [c, z] if case["preact"] else [c]
    if case["op"] == "activation_grad":
        z = s["Z"]
        if case["act"] == "relu":
            slope = torch.sign(z).clamp(min=0.0)
        elif case["act"] == "gelu":
            slope = 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
        elif case["act"] == "gelu_tanh":
            a = 2.0 * math.sqrt(2.0 / math.pi)
            p = torch.sigmoid(a * (z + 0.044715 * z ** 3))
            slope = p + z * p * (1.0 - p) * a * (1.0 + 0.134145 * z ** 2)
        elif case["act"] == "silu":
            p = torch.sigmoid(z)
            slope = p + z * p * (1.0 - p)
        else:
            slope = torch.ones_like(z)
        dZ = slope * s["dC"]
        return [dZ, dZ.sum(dim=0)] if case["bias"] else [dZ]

    def deviation(x):
        mean = x.sum(1, keepdim=True) / x.shape[1] if case["kind"] == "layer" else torch.zeros_like(x[:, :1])
        return mean, torch.rsqrt(((x - mean) ** 2).sum(1, keepdim=True) / x.shape[1] + 1e-5)

    def through(x, grad):
        """The gradient of sum(grad * standardised x) with respect to x."""
        mean, r = deviation(x)
        z, n = (x - mean) * r, x.shape[1]
        inner = (grad * z).sum(1, keepdim=True) / n
        shift = grad.sum(1, keepdim=True) / n if case["kind"] == "layer" else 0.0
        return r * (grad - shift - z * inner), z
    gate = None
    if case["post"]:
        gate = torch.ones((1, 1), dtype=torch.float64, device="cuda") if s["gate"] is None else s["gate"][:, None] if case["gate"] == "row" else s["gate"]
    if case["op"] == "norm":
        h, out = s["H"], []
        if case["post"]:
            mean, r = deviation(s["Y"])
            v = (s["Y"] - mean) * r * s["post_weight"]
            if s["post_bias"] is not None:
                v = v + s["post_bias"]
            h = case["alpha"] * h + gate * v
            out.append(h)
        if case["pre"]:
            mean, r = deviation(h)
            n = (h - mean) * r * s["pre_weight"]
            out.append(n if s["pre_bias"] is None else n + s["pre_bias"])
        return out
    d, sums = s["dH_out"], []
    if case["pre"]:
        back, z = through(s["H"], s["dn"] * s["pre_weight"])
        d = d + back
        sums.append((z * s["dn"]).sum(0))
        if s["pre_bias"] is not None:
            sums.append(s["dn"].sum(0))
    if not case["post"]:
        return [d] + sums
    dv = gate * d
    dY, z = through(s["Y"], dv * s["post_weight"])
    sums.append((z * dv).sum(0))
    if s["post_bias"] is not None:
        sums.append(dv.sum(0))
    if s["gate"] is not None:
        v = z * s["post_weight"] + (0.0 if s["post_bias"] is None else s["post_bias"])
        dg = d * v
        sums.append(dg.sum(1) if case["gate"] == "row" else dg.sum(0) if case["gate"] == "col" else dg)
    return [case["alpha"] * d] + sums + [dY]
