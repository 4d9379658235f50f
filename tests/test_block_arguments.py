"""What the operators around the product refuse, on the host, before any device call."""
import ctypes

import pytest
import torch

import paper_2402_14118_amd as mm
from paper_2402_14118_amd import binding as B

AT = 0x7000_0000_0000          # never dereferenced on the host


def at(i):
    return AT + (i << 32)


def norm(desc, h=at(0), ldh=64, y=None, ldy=0, gate=None, ldgate=0, pw=None, pb=None, w=None, b=None, h_out=None, ldho=0, n=at(1), ldn=64):
    return B.lib.mmm_block_norm(None if desc is None else ctypes.byref(desc), h, ldh, y, ldy, gate, ldgate, pw, pb, w, b, h_out, ldho, n, ldn, None)


def desc(M=4, N=64, dt=0, dt_h=0, dt_y=0, post=0, pre=1, gate=0, eps=1e-5, alpha=1.0):
    return mm.BlockNormDesc(M, N, dt, dt_h, dt_y, post, pre, gate, eps, alpha)


def test_norm_refuses():
    assert norm(None) == B.MMM_ERR_INVALID_ARG
    for bad in (dict(dt=3), dict(dt=9), dict(dt_h=1), dict(dt_y=2), dict(dt=1, dt_h=2), dict(dt=1, dt_h=3)):
        assert norm(desc(**bad)) == B.MMM_ERR_DTYPE, bad
    for bad in (dict(M=0), dict(N=0), dict(N=mm.MMM_NORM_MAX_WIDTH + 1), dict(M=(1 << 30) + 1)):
        assert norm(desc(**bad), ldh=1 << 20, ldn=1 << 20) == B.MMM_ERR_SHAPE, bad
    for bad in (dict(post=3), dict(pre=-1), dict(gate=4), dict(eps=-1.0), dict(eps=float("nan"))):
        assert norm(desc(**bad)) == B.MMM_ERR_INVALID_ARG, bad
    d, both = desc(), desc(post=1, gate=2)
    assert norm(d, h=None) == norm(d, n=None) == norm(desc(pre=0)) == B.MMM_ERR_INVALID_ARG
    # no block: nothing behind it
    assert norm(d, h_out=at(2), ldho=64) == norm(desc(post=1)) == norm(desc(gate=1), gate=at(2)) == B.MMM_ERR_INVALID_ARG
    assert norm(d, pw=at(2)) == norm(desc(pre=0), y=at(2), ldy=64, h_out=at(3), ldho=64, n=None, w=at(4)) == B.MMM_ERR_INVALID_ARG
    # the gate that is announced, and no other
    assert norm(both, y=at(2), ldy=64) == norm(desc(post=1), y=at(2), ldy=64, gate=at(3)) == B.MMM_ERR_INVALID_ARG
    assert norm(d, ldh=63) == norm(d, ldn=63) == norm(both, y=at(2), ldy=63, gate=at(3)) == B.MMM_ERR_SHAPE
    assert norm(desc(post=1, gate=3), y=at(2), ldy=64, gate=at(3), ldgate=63) == B.MMM_ERR_SHAPE
    assert norm(both, y=at(2), ldy=64, gate=at(3), h_out=at(0), ldho=65) == B.MMM_ERR_SHAPE      # in place is in place
    assert norm(d, h=at(0) + 2) == norm(d, w=at(2) + 1) == norm(both, y=at(2), ldy=64, gate=at(3) + 2) == B.MMM_ERR_DTYPE


def grads(d, ws=at(20), nbytes=1 << 30, **k):
    g = mm.BlockNormGrads()
    for name, v in k.items():
        setattr(g, name, v)
    return B.lib.mmm_block_norm_backward(ctypes.byref(d), ctypes.byref(g), ws, nbytes, None)


def test_norm_backward_refuses():
    full = dict(h_out=at(0), ldh_out=64, y=at(1), ldy=64, gate_values=at(2), d_n=at(3), ldd_n=64, d_h=at(4), ldd_h=64, d_pre_weight=at(5))
    d = desc(post=1, gate=2)
    assert B.lib.mmm_block_norm_backward(ctypes.byref(d), None, None, 0, None) == B.MMM_ERR_INVALID_ARG
    # with what is asked for nothing missing, a workspace that is too small is what is left to refuse
    assert grads(d, nbytes=16, **full) == B.MMM_ERR_WORKSPACE
    assert grads(d, ws=None, **full) == grads(d, ws=at(20) + 8, **full) == B.MMM_ERR_WORKSPACE
    assert grads(d, nbytes=mm.mmm_block_norm_backward_workspace_bytes(4, 64) - 256, **full) == B.MMM_ERR_WORKSPACE

    def without(*names, **more):
        return grads(d, nbytes=16, **{k: v for k, v in full.items() if k not in names}, **more)
    for missing in ("h_out", "y", "gate_values", "d_n"):
        assert without(missing) == B.MMM_ERR_INVALID_ARG, missing
    assert without("d_h", "d_pre_weight") == B.MMM_ERR_INVALID_ARG        # nothing asked for
    assert without("ldh_out") == without("ldd_n") == without("ldd_h") == without("ldy") == B.MMM_ERR_SHAPE
    assert without(d_h_out=at(4), ldd_h_out=65) == B.MMM_ERR_SHAPE
    assert without("d_pre_weight", d_pre_weight=at(5) + 2) == B.MMM_ERR_DTYPE
    # no norm in front: its operands are not taken, and a gradient has to come in
    p = desc(post=1, pre=0)
    assert grads(p, y=at(1), ldy=64, d_y=at(4), ldd_y=64) == B.MMM_ERR_INVALID_ARG
    assert grads(p, y=at(1), ldy=64, d_y=at(4), ldd_y=64, d_h_out=at(5), ldd_h_out=64, d_pre_bias=at(6)) == B.MMM_ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    assert B.lib.mmm_block_norm_backward_workspace_bytes(0, 8, ctypes.byref(n)) == B.MMM_ERR_SHAPE
    assert B.lib.mmm_block_norm_backward_workspace_bytes(8, 40000, ctypes.byref(n)) == B.MMM_ERR_SHAPE
    assert B.lib.mmm_block_norm_backward_workspace_bytes(8, 8, None) == B.MMM_ERR_INVALID_ARG


def test_epilogue_backward_refuses():
    def call(M=4, N=16, dt=1, out=1, act=1, dC=at(0), lddc=16, Z=at(1), ldz=16, dZ=at(2), lddz=16, db=None, ws=None, n=0):
        return B.lib.mmm_epilogue_backward(M, N, dt, out, act, dC, lddc, Z, ldz, dZ, lddz, db, ws, n, None)
    assert call(act=5) == call(act=-1) == call(dC=None) == call(Z=None) == call(dZ=None) == B.MMM_ERR_INVALID_ARG
    assert call(dt=3, out=3) == call(dt=1, out=2) == call(dt=0, out=1) == call(dt=4) == B.MMM_ERR_DTYPE
    assert call(M=0) == call(N=0) == call(lddc=15) == call(ldz=15) == call(lddz=15) == B.MMM_ERR_SHAPE
    assert call(dC=at(0) + 1) == call(Z=at(1) + 1) == call(dZ=at(2) + 1) == call(db=at(3) + 2, ws=at(4), n=1 << 20) == B.MMM_ERR_DTYPE
    need = mm.mmm_epilogue_backward_workspace_bytes(4, 16)
    assert call(db=at(3)) == call(db=at(3), ws=at(4), n=need - 1) == call(db=at(3), ws=at(4) + 128, n=need) == B.MMM_ERR_WORKSPACE
    n = ctypes.c_size_t(0)
    assert B.lib.mmm_epilogue_backward_workspace_bytes(0, 1, ctypes.byref(n)) == B.MMM_ERR_SHAPE
    assert B.lib.mmm_epilogue_backward_workspace_bytes(1, 1, None) == B.MMM_ERR_INVALID_ARG


def test_epilogue_backward_in_place_is_in_place():
    """dZ at the address of dC or Z, with rows or elements of another size."""
    def call(dZ, lddz, dt=1, act=1, lddc=16, ldz=16):
        return B.lib.mmm_epilogue_backward(4, 16, dt, 0, act, at(0), lddc, at(1), ldz, dZ, lddz, None, None, 0, None)
    assert call(at(0), 17, dt=0) == call(at(1), 17, dt=0) == call(at(1), 16, dt=0, ldz=17) == B.MMM_ERR_SHAPE
    assert call(at(0), 16) == call(at(1), 16) == B.MMM_ERR_DTYPE


def test_the_holder_checks_tensors():
    norm = mm.BlockNorm(4, 16, mm.MMM_BF16, post=mm.MMM_NORM_RMS, gate=mm.MMM_GATE_ROW, device="cpu")
    H = torch.zeros(4, 16, dtype=torch.bfloat16)
    for bad, error in ((dict(H=H[:3]), ValueError), (dict(H=H.float()), TypeError), (dict(H=H.t().contiguous().t()), ValueError), (dict(H=None), ValueError),
                       (dict(Y=H[:, :8]), ValueError), (dict(gate=torch.zeros(16, dtype=torch.bfloat16)), ValueError), (dict(pre_weight=torch.zeros(16)), TypeError)):
        with pytest.raises(error):
            norm.forward(**{"H": H, "normed": torch.empty_like(H), **bad})
    with pytest.raises(mm.MmmError):
        mm.BlockNorm(0, 16, device="cpu")
    with pytest.raises(ValueError):
        mm.BlockNorm(4, 16, mm.MMM_BF16, device="cpu").forward(H, normed=torch.empty_like(H), gate=H[0])


def test_matmul_epilogue_refuses():
    need = mm.mmm_maps_workspace_bytes(64, 128, 64, 16)
    maps = mm.mmm_maps_init(AT, need, 64, 128, 64, 16)
    ma = mm.MaskA(0, 0.0, None)

    def call(dt=1, X=at(1), ldx=128, mask=None, Y=at(2), ldy=64, C=at(3), ldc=64, e="default", handle=maps, **k):
        e = mm.Epilogue(**{"activation": 1, "out_dtype": dt, **k}) if e == "default" else e
        return B.lib.mmm_matmul_epilogue(handle, dt, X, ldx, None if mask is None else ctypes.byref(mask), Y, ldy, C, ldc, None if e is None else ctypes.byref(e), None)
    try:
        for mask in (None, ma):
            assert call(mask=mask) == B.MMM_ERR_MAPS_MISMATCH       # nothing is built: what is refused below is refused before that
            assert call(mask=mask, e=None) == call(mask=mask, C=None) == call(mask=mask, handle=None) == B.MMM_ERR_INVALID_ARG
            assert call(mask=mask, activation=5) == call(mask=mask, activation=-1) == B.MMM_ERR_INVALID_ARG
            assert call(mask=mask, out_dtype=2) == call(mask=mask, out_dtype=3) == call(mask=mask, dt=3, out_dtype=0) == B.MMM_ERR_DTYPE
            assert call(mask=mask, dt=0, out_dtype=1) == call(mask=mask, out_dtype=7) == B.MMM_ERR_DTYPE
            assert call(mask=mask, out_dtype=0) == call(mask=mask, dt=3, Y=at(2)) == B.MMM_ERR_MAPS_MISMATCH
            assert call(mask=mask, ldc=63) == call(mask=mask, residual=at(4), ldr=63) == call(mask=mask, preact=at(4), ldp=63) == B.MMM_ERR_SHAPE
            assert call(mask=mask, residual=at(3), ldr=65) == B.MMM_ERR_SHAPE                   # in place is in place
            assert call(mask=mask, bias=at(4) + 1) == call(mask=mask, residual=at(4) + 1, ldr=64) == call(mask=mask, preact=at(4) + 1, ldp=64) == B.MMM_ERR_DTYPE
            assert call(mask=mask, C=at(3) + 1) == call(mask=mask, C=at(3) + 2, out_dtype=0) == B.MMM_ERR_DTYPE
            assert call(mask=mask, C=at(3) + 2) == B.MMM_ERR_MAPS_MISMATCH                      # a 16-bit C starts at any of its elements
        assert call(mask=mm.MaskA(3, 0.0, None)) == call(mask=mm.MaskA(0, 0.0, at(5) + 4)) == B.MMM_ERR_INVALID_ARG
    finally:
        mm.mmm_maps_release(maps)


def test_the_engine_checks_tensors_of_the_epilogue():
    eng = object.__new__(mm.MaskedMatmul)
    eng.M, eng.K, eng.N, eng.dtype, eng.device, eng.maps = 4, 8, 16, mm.MMM_BF16, torch.device("cpu"), None
    h = torch.bfloat16
    X, Y, C = torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)
    for bad, error in ((dict(X=X.float()), TypeError), (dict(Y=Y[:4]), ValueError), (dict(bias=C[0].float()), TypeError),
                       (dict(bias=C[0, :8]), ValueError), (dict(residual=C.float()), TypeError), (dict(preact=C[:2]), ValueError),
                       (dict(C=torch.zeros(16, 4, dtype=h).t()), ValueError)):
        with pytest.raises(error):
            eng.matmul_epilogue(**{"X": X, "Y": Y, "C": C, **bad}, stream=0)
    with pytest.raises(mm.MmmError) as e:
        eng.matmul_epilogue(X, Y, C, stream=0)
    assert e.value.status == B.MMM_ERR_INVALID_ARG


def test_matmul_backward_refuses():
    need = mm.mmm_maps_workspace_bytes(64, 128, 64, 16)
    maps = mm.mmm_maps_init(AT, need, 64, 128, 64, 16)

    def call(handle=maps, dt=1, X=at(1), ldx=128, Y=at(2), ldy=64, dC=at(3), lddc=64, dX=at(4), lddx=128, dY=at(5), lddy=64):
        return B.lib.mmm_matmul_backward(handle, dt, X, ldx, Y, ldy, dC, lddc, dX, lddx, dY, lddy, 0, 0, None)
    try:
        assert call() == call(dX=None, lddx=0) == call(dY=None, lddy=0) == B.MMM_ERR_MAPS_MISMATCH
        for missing in (dict(handle=None), dict(X=None), dict(Y=None), dict(dC=None), dict(dX=None, dY=None)):
            assert call(**missing) == B.MMM_ERR_INVALID_ARG
        assert call(dt=3) == call(dt=4) == call(X=at(1) + 1) == call(dC=at(3) + 1) == call(dX=at(4) + 1) == call(dY=at(5) + 2) == B.MMM_ERR_DTYPE
        for short in (dict(ldx=127), dict(ldy=63), dict(lddc=63), dict(lddx=127), dict(lddy=63), dict(lddc=1 << 22)):
            assert call(**short) == B.MMM_ERR_SHAPE
    finally:
        mm.mmm_maps_release(maps)


class Recorder:
    """Stands for a product: notes what is called."""

    def __init__(self, calls):
        self.calls = calls

    def __getattr__(self, name):
        return lambda *args, **kwargs: self.calls.append(name)


def mlp_of(calls, M=4, width=16, hidden=32, dtype=mm.MMM_F32, device="cpu", **more):
    """A holder whose products only note that they were called."""
    mlp = object.__new__(mm.MaskedMlp)
    t = torch.float32 if dtype == mm.MMM_F32 else torch.bfloat16
    room = {name: torch.zeros(M, n, dtype=t) for name, n in (("a", hidden), ("y", width), ("grad_a", hidden), ("grad_y", width))}
    mlp.__dict__.update(M=M, width=width, hidden=hidden, dtype=dtype, activation=mm.MMM_ACT_RELU, fused=False, training=True, device=torch.device(device),
                        up=Recorder(calls), down=Recorder(calls), norm=mm.BlockNorm(M, width, dtype, mm.MMM_NORM_RMS, device="cpu", training=True),
                        preact=room["a"], W1=torch.zeros(width, hidden, dtype=t), W2=torch.zeros(hidden, width, dtype=t), b1=None, b2=None, masks=({}, {}), counted=False,
                        workspace=torch.empty(1 << 16, dtype=torch.uint8), **room)
    mlp.norm.device = mlp.device
    mlp.__dict__.update(more)
    return mlp


def test_the_block_refuses_another_current_device_before_any_launch(monkeypatch):
    """Every product of it would be launched there."""
    calls = []
    mlp = mlp_of(calls, device="cuda:1")
    monkeypatch.setattr(B, "current_device", lambda: 0)
    monkeypatch.setattr("paper_2402_14118_amd.block.places", lambda *a: (None, 0) * 20)
    N = torch.zeros(4, 16)
    for call in (lambda: mlp.forward(N, N, N, N), lambda: mlp.count()):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert calls == []


def test_the_block_refuses_operands_before_any_launch(monkeypatch):
    """A call that cannot be carried out to its end is not begun: with accumulate the weights' gradients have been added to by then."""
    calls = []
    mlp = mlp_of(calls, built=None)
    for name in ("block_norm", "block_norm_backward", "epilogue_backward"):
        monkeypatch.setattr(B.native, name, lambda *a, name=name: calls.append(name) or 0)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    N, w1, w2 = torch.zeros(4, 16), torch.zeros(16, 32), torch.zeros(32, 16)
    H, out, n = (torch.zeros(4, 16) for _ in range(3))
    good = dict(N=N, H_out=out, grad_N=torch.zeros(4, 16), grad_H=H, grad_normed=n, grad_W1=w1, grad_W2=w2, grad_b1=torch.zeros(32), accumulate=True)
    with pytest.raises(ValueError, match="forward"):
        mlp.backward(**good)                                     # there was none
    for bad in (dict(H=H[:3]), dict(H_out=out.double()), dict(normed=n[:, :8]), dict(gate=N), dict(pre_weight=N), dict(N=N[:2])):
        with pytest.raises((ValueError, TypeError)):
            mlp.forward(**{"N": N, "H": H, "H_out": out, "normed": n, **bad})
    assert calls == []
    mlp.forward(N, H, out, n)
    assert calls == ["build_maps", "matmul_epilogue", "build_maps", "matmul_epilogue", "block_norm"]
    calls.clear()
    for bad in (dict(N=N.clone()), dict(N=N[:2]), dict(grad_N=H[:2]), dict(grad_W1=w2), dict(grad_W1=w1.double()), dict(grad_W2=w1), dict(grad_b1=torch.zeros(16)),
                dict(grad_b2=torch.zeros(32)), dict(grad_N=None, grad_W1=None), dict(grad_W2=torch.zeros(1, 16).expand(32, 16)), dict(grad_H=H[:2])):
        with pytest.raises((ValueError, TypeError)):
            mlp.backward(**{**good, **bad})
    assert calls == []
    mlp.backward(**good)
    assert calls == ["block_norm_backward", "matmul_backward", "epilogue_backward", "matmul_backward"]


@pytest.mark.parametrize("dtype", [mm.MMM_F64, 7])
def test_the_block_refuses_types_without_norms(dtype):
    """At once, not behind the products of the first call."""
    with pytest.raises(ValueError, match="floats"):
        mm.MaskedMlp(4, 64, 64, dtype=dtype, device="cpu")


def test_a_mask_without_a_predicate_is_refused():
    """Without a predicate the maps say what counts: a mask that is given would be left out."""
    eng = object.__new__(mm.MaskedMatmul)
    eng.M, eng.K, eng.N, eng.dtype, eng.device, eng.maps = 4, 8, 16, mm.MMM_BF16, torch.device("cpu"), None
    X, Y, C = (torch.zeros(s, dtype=torch.bfloat16) for s in ((4, 8), (8, 16), (4, 16)))
    for mask in (dict(keep_a=torch.zeros(4, 1, dtype=torch.int64)), dict(threshold=0.5)):
        with pytest.raises(ValueError, match="predicate"):
            eng.matmul_epilogue(X, Y, C, stream=0, **mask)
