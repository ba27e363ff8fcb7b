"""Refusals of the 4-bit and grouped calls, which come before any device access, and their sizes.  No GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2505_14742_amd import binding as q

A = 0x1000      # a non-null, 16-byte aligned fake device address


def _call(name, defaults, **change):
    args = {**defaults, **change}
    assert set(args) == set(defaults)
    return getattr(q.lib(), name)(*[C.c_float(v) if isinstance(v, float) else v for v in args.values()])


MX4 = dict(X=A, t=8, ldx=64, offsets=A, n_groups=3, codes=A, scales=A, c_in=64, c_out=64, lora_A=A, lora_B=A, r=16, scale=1.0, Y=A, ldy=64,
           ws=A, bytes=1 << 20, stream=None)
ROWS = dict(X=A, t=8, ldx=64, offsets=A, n_groups=3, W=A, c_in=64, c_out=64, scale=1.0, accumulate=0, Y=A, ldy=64, ws=A, bytes=1 << 20, stream=None)
DW = dict(X=A, ldx=64, dY=A, lddy=64, t=8, offsets=A, n_groups=3, c_in=64, c_out=64, scale=1.0, dW=A, ws=A, bytes=1 << 20, stream=None)


@pytest.mark.parametrize("name", ["quaff_mx4_linear_fwd", "quaff_mx4_linear_fwd_bf16", "quaff_mx4_linear_bwd_dx", "quaff_mx4_linear_bwd_dx_bf16"])
def test_mx4_linear_refusals(name):
    refused = lambda want, **change: _call(name, MX4, **change) == want
    for key in ("X", "codes", "scales", "lora_A", "lora_B", "Y"):
        assert refused(q.ERR_NULL, **{key: None}), key
        assert refused(q.ERR_ALIGN, **{key: A + 8}), key
    for change in (dict(t=-1), dict(t=1 << 30), dict(c_in=72), dict(c_out=8), dict(c_out=1 << 20), dict(r=8), dict(r=80), dict(ldx=48), dict(ldy=48),
                   dict(ldx=1 << 22), dict(ldy=1 << 27), dict(n_groups=0), dict(n_groups=1025), dict(n_groups=-1), dict(offsets=None)):
        assert refused(q.ERR_SHAPE, **change), change
    assert refused(q.ERR_ALIGN, ldx=68) and refused(q.ERR_ALIGN, offsets=A + 4) and refused(q.ERR_ALIGN, ws=A + 8)
    assert refused(q.ERR_ALIGN, ldy=66)
    assert refused(q.ERR_WORKSPACE, ws=None) and refused(q.ERR_WORKSPACE, bytes=100)
    assert refused(q.OK, t=0, X=None, Y=None, ws=None)              # nothing to do


@pytest.mark.parametrize("name", ["quaff_grouped_linear_fwd", "quaff_grouped_linear_fwd_bf16", "quaff_grouped_linear_bwd_dx",
                                  "quaff_grouped_linear_bwd_dx_bf16"])
def test_grouped_linear_refusals(name):
    defaults = {k: v for k, v in ROWS.items() if not (k == "accumulate" and name.endswith("bf16"))}
    refused = lambda want, **change: _call(name, defaults, **change) == want
    for key in ("X", "W", "Y", "offsets"):
        assert refused(q.ERR_NULL, **{key: None}), key
        assert refused(q.ERR_ALIGN, **{key: A + 4}), key
    for change in (dict(t=-1), dict(t=1 << 30), dict(c_in=72), dict(c_in=0), dict(c_out=8), dict(ldx=48), dict(ldy=48), dict(ldx=1 << 22),
                   dict(ldy=1 << 27), dict(n_groups=0), dict(n_groups=1025)):
        assert refused(q.ERR_SHAPE, **change), change
    assert refused(q.ERR_ALIGN, ldx=68) and refused(q.ERR_ALIGN, ldy=66)
    assert refused(q.OK, t=0, X=None, Y=None)


def test_weight_gradient_refusals():
    refused = lambda want, **change: _call("quaff_grouped_linear_bwd_dw", DW, **change) == want
    for key in ("X", "dY", "dW", "offsets"):
        assert refused(q.ERR_NULL, **{key: None}), key
        assert refused(q.ERR_ALIGN, **{key: A + 4}), key
    for change in (dict(t=-1), dict(c_in=72), dict(c_out=8), dict(ldx=48), dict(lddy=48), dict(ldx=1 << 22), dict(n_groups=0), dict(n_groups=1025)):
        assert refused(q.ERR_SHAPE, **change), change
    assert refused(q.ERR_ALIGN, ldx=68) and refused(q.ERR_ALIGN, lddy=68)


def test_quantizer_refusals():
    quant = dict(X=A, rows=8, k=64, ldx=64, codes=A, scales=A, stream=None)
    deq = dict(codes=A, scales=A, rows=8, k=64, out=A, ldo=64, stream=None)
    prep = dict(W=A, n=1, c_in=64, c_out=64, ldw=64, cf=A, sf=A, cb=A, sb=A, stream=None)
    for name, d in (("quaff_mx4_quantize", quant), ("quaff_mx4_dequantize", deq)):
        for key in [k for k, v in d.items() if v == A]:
            assert _call(name, d, **{key: None}) == q.ERR_NULL and _call(name, d, **{key: A + 8}) == q.ERR_ALIGN
        ld = "ldx" if "ldx" in d else "ldo"
        for change in (dict(rows=-1), dict(rows=1 << 30), dict(k=40), dict(k=0), {ld: 48}):
            assert _call(name, d, **change) == q.ERR_SHAPE, change
        assert _call(name, d, **{ld: 68}) == q.ERR_ALIGN
        assert _call(name, d, rows=0) == q.OK
    p = lambda **change: _call("quaff_mx4_prepare_weight", prep, **change)
    assert p(W=None) == p(sf=None) == p(cb=None) == p(cf=None, sf=None, cb=None, sb=None) == q.ERR_NULL
    assert p(n=0) == p(n=1025) == p(c_in=40) == p(c_out=0) == p(ldw=48) == q.ERR_SHAPE
    assert p(W=A + 4) == p(cf=A + 8) == p(sb=A + 8) == p(ldw=66) == q.ERR_ALIGN


def test_offset_check_refusals():
    chk = lambda offsets=A, n=3, t=8, res=A: q.lib().quaff_check_group_offsets(offsets, n, t, res, None)
    assert chk(offsets=None) == chk(res=None) == q.ERR_NULL
    assert chk(n=0) == chk(n=1025) == chk(t=-1) == q.ERR_SHAPE
    assert chk(offsets=A + 4) == chk(res=A + 2) == q.ERR_ALIGN


def test_sizes():
    for k, kp in ((-3, 0), (0, 0), (1, 256), (256, 256), (257, 512), (1040, 1280)):
        assert q.mx4_padded(k) == q.lib().quaff_mx4_padded(k) == kp
    small, large = q.mx4_linear_workspace_bytes(100, 1024, 2048, 0, 16), q.mx4_linear_workspace_bytes(200, 1024, 2048, 0, 16)
    assert 100 * 2048 * 17 // 32 + 100 * 16 * 4 <= small < large
    assert q.mx4_linear_workspace_bytes(100, 1024, 2048, 0, 0) == q.mx4_linear_workspace_bytes(100, 2048, 1024, 0, 0)
    assert q.mx4_linear_workspace_bytes(-1, 64, 64, 0, 0) == 0 and q.grouped_linear_workspace_bytes(-1, 64, 64, 1) == 0


def test_the_binding_refuses_tensors_of_another_device():
    X, W, off = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, 64, 48, dtype=torch.bfloat16), torch.tensor([0, 1, 4])
    with pytest.raises(q.QuaffError):
        q.grouped_linear_fwd(X, off, W, 1.0, torch.zeros(4, 48), None)
    with pytest.raises(q.QuaffError):
        q.mx4_quantize(X, torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8))


def test_the_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    """Sizes and types that the C entries, which see pointers only, cannot check; before any device access."""
    monkeypatch.setattr(q, "_where", lambda t: t.get_device())
    X, W = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, 64, 48, dtype=torch.bfloat16)
    off, Y, ws = torch.tensor([0, 1, 4]), torch.zeros(4, 48), torch.zeros(1 << 16, dtype=torch.int8)
    codes, scales = torch.zeros(96, 128, dtype=torch.uint8), torch.zeros(96, 8, dtype=torch.uint8)
    bad = [lambda: q.grouped_linear_fwd(X.float(), off, W, 1.0, Y, ws), lambda: q.grouped_linear_fwd(X, off.int(), W, 1.0, Y, ws),
           lambda: q.grouped_linear_fwd(X, off[:2], W, 1.0, Y, ws), lambda: q.grouped_linear_fwd(X, off, W, 1.0, Y[:3], ws),
           lambda: q.grouped_linear_fwd(X, off, W, 1.0, Y, ws, bf16_out=True), lambda: q.grouped_linear_fwd(X[:, :48], off, W, 1.0, Y, ws),
           lambda: q.grouped_linear_fwd(X, off, W, 1.0, Y.to(torch.bfloat16), ws, bf16_out=True, accumulate=True),
           lambda: q.grouped_linear_bwd_dx(X, off, W, 1.0, Y, ws), lambda: q.grouped_linear_bwd_dw(X, X[:3], off, 1.0, torch.zeros(2, 64, 64), ws),
           lambda: q.grouped_linear_bwd_dw(X, X, off, 1.0, torch.zeros(2, 64, 48), ws), lambda: q.mx4_quantize(X, codes[:3], scales),
           lambda: q.mx4_quantize(X.t(), codes, scales), lambda: q.mx4_dequantize(codes[:3], scales, X),
           lambda: q.mx4_linear_fwd(X, off, codes[:95], scales, 64, 48, None, None, 0, 1.0, Y, ws),
           lambda: q.mx4_linear_fwd(X, off, codes, scales[:95], 64, 48, None, None, 0, 1.0, Y, ws),
           lambda: q.mx4_linear_fwd(X, off, codes, scales, 64, 48, X, X, 16, 1.0, Y, ws),
           lambda: q.mx4_linear_fwd(X, off, codes, scales, 64, 48, None, None, 16, 1.0, Y, ws),
           lambda: q.mx4_prepare_weight(torch.zeros(64, 48), codes, scales, codes[:63], scales)]
    for i, call in enumerate(bad):
        with pytest.raises(q.QuaffError) as e:
            call()
        assert e.value.status == q.ERR_SHAPE, i


def test_every_form_has_sizes_of_its_own():
    """The kernel forms that the GPU tests of these products are meant to reach (their sizes, or near them), and the rules' two sides."""
    form = q.debug_group_form
    assert form("mx4_fwd", 1, 4096, 1040, 0) == form("dx", 20, 2048, 1408, 64) == form("fwd", 700, 2048, 1408, 64) == "few rows"
    assert form("mx4_fwd", 150, 2048, 1408, 64) == form("dx", 700, 2048, 1408, 64) == form("fwd", 586, 64, 3776, 243) == "64x64"
    for what in ("mx4_fwd", "fwd"):
        assert form(what, 3833, 528, 1168, 40) == "128x128" and form(what, 4106, 592, 4112, 2) == "256x256", what
    for what in ("mx4_dx", "dx"):
        assert form(what, 3833, 1168, 592, 40) == "128x128" and form(what, 4106, 4112, 528, 2) == "256x256", what
    assert form("fwd", 842, 4112, 16, 4) == form("dx", 842, 48, 4112, 4) == form("mx4_dx", 3466, 256, 14848, 0) == "64x64 parts"
    dw = {(9009, 208, 16, 2): "128x32 slabs", (513, 208, 16, 1): "128x32 slabs", (200, 208, 16, 3): "128x32", (3413, 272, 64, 3): "128x64 slabs",
          (100, 272, 48, 2): "128x64", (9000, 16, 400, 1): "32x128 slabs", (90, 16, 400, 2): "32x128", (3030, 64, 2064, 4): "64x128 slabs",
          (100, 64, 2064, 4): "64x128", (3042, 400, 272, 3): "128x128 slabs", (90, 272, 400, 3): "128x128", (1029, 1040, 1040, 16): "256x256"}
    for (t, c_in, c_out, n), want in dw.items():
        assert form("dw", t, c_in, c_out, n) == want, (t, c_in, c_out, n, form("dw", t, c_in, c_out, n))
    assert q.lib().quaff_debug_group_form(5, 8, 64, 64, 1) == q.lib().quaff_debug_group_form(2, 8, 64, 64, 0) == b""
