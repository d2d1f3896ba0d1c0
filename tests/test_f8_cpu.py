"""The e4m3 entry points and the norms without a GPU: what they refuse, in which
order and with which code, the workspaces they ask for, and the binding's own checks."""
import ctypes as C

import pytest
import torch

from paper_2606_15177_amd import workloads as W
from tests.test_gpu_f8 import FEW, FFN_KERNELS

F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def moe():
    from paper_2606_15177_amd import moe
    return moe


@pytest.mark.parametrize("rows,cols,x,ldx,q,ldq,scale,code", [
    (-1, 8, 16, 8, 16, 16, 16, -2), (4, 0, 16, 8, 16, 16, 16, -2), (4, 8, 16, 7, 16, 16, 16, -2),
    (4, 33, 16, 33, 16, 32, 16, -2),                       # ldq below cols
    (4, 8, 16, 8, 16, 24, 16, -6), (4, 8, 17, 8, 16, 16, 16, -6), (4, 8, 16, 8, 24, 16, 16, -6),
    (4, 8, 16, 8, 16, 16, 18, -6), (4, 8, None, 8, 16, 16, 16, -1), (4, 8, 16, 8, None, 16, 16, -1),
    (4, 8, 16, 8, 16, 16, None, -1), (4, 8, 16, 2 ** 41, 16, 16, 16, -3), (4, 2 ** 31 - 1, 16, 2 ** 31, 16, 2 ** 31, 16, -3),
    (0, 8, None, 8, None, 16, None, 0),                    # no rows: nothing to do
])
def test_quantize_refusals(moe, rows, cols, x, ldx, q, ldq, scale, code):
    assert moe._lib.moe_quantize_rows_f8(rows, cols, x, ldx, q, ldq, scale, None) == code
    # no rows of no matrices is nothing to do, no rows of a matrix is none
    g, r = (0, 4) if rows == 0 else (2, rows)
    assert moe._lib.moe_quantize_blocks_f8(g, r, cols, x, ldx, q, ldq, scale, None) == code


def test_quantize_blocks_refusals(moe):
    f = moe._lib.moe_quantize_blocks_f8
    assert f(-1, 4, 8, 16, 8, 16, 16, 16, None) == moe.MOE_ERR_DIMS
    assert f(1, 0, 8, 16, 8, 16, 16, 16, None) == moe.MOE_ERR_DIMS
    assert f(2 ** 17, 2 ** 14, 128, 16, 128, 16, 128, 16, None) == moe.MOE_ERR_UNSUPPORTED   # workgroups: 2^24


LIN = dict(M=4, N=8, K=40, G=2, X=4, ldx=48, ldw=48, ldy=8)


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), -2), (dict(N=0), -2), (dict(K=0), -2), (dict(ldx=32), -2), (dict(ldw=32), -2), (dict(ldy=7), -2),
    (dict(ldx=56), -6), (dict(ldw=56), -6), (dict(K=2 ** 17, ldx=2 ** 17, ldw=2 ** 17), -3), (dict(ldx=2 ** 21 + 16), -3),
    (dict(ldw=2 ** 21 + 16), -3), (dict(ldy=2 ** 21 + 1), -3), (dict(N=2 ** 24 + 1, ldy=2 ** 25), -3), (dict(M=0), 0),
    (dict(M=2 ** 31 - 200), -3),
])
def test_linear_refusals(moe, change, code):
    d = moe.MoeLinearDims(**{**LIN, **change})
    assert moe._lib.moe_linear_f8(C.byref(d), 16, 16, 16, 16, 16 if code else None, None) == code
    assert moe._lib.moe_grouped_linear_f8(C.byref(d), 16, 16, None, 16, 16, 16, 16 if code else None, None) == code


@pytest.mark.parametrize("ptrs,code", [
    ((None, 16, 16, 16, 16), -1), ((16, None, 16, 16, 16), -1), ((16, 16, None, 16, 16), -1), ((16, 16, 16, None, 16), -1),
    ((16, 16, 16, 16, None), -1), ((24, 16, 16, 16, 16), -6), ((16, 18, 16, 16, 16), -6), ((16, 16, 24, 16, 16), -6),
    ((16, 16, 16, 18, 16), -6), ((16, 16, 16, 16, 17), -6),
])
def test_linear_pointers(moe, ptrs, code):
    d = moe.MoeLinearDims(**LIN)
    xq, xs, wq, ws, y = ptrs
    assert moe._lib.moe_linear_f8(C.byref(d), xq, xs, wq, ws, y, None) == code
    assert moe._lib.moe_grouped_linear_f8(C.byref(d), xq, xs, None, 16, wq, ws, y, None) == code
    assert moe._lib.moe_linear_f8(None, xq, xs, wq, ws, y, None) == moe.MOE_ERR_NULL


@pytest.mark.parametrize("change,x_rows,offsets,code", [
    (dict(G=0), None, 16, -2), (dict(G=1025), None, 16, -3), (dict(X=-1), 16, 16, -2), (dict(), None, None, -1),
    (dict(), 18, 16, -6), (dict(), 16, 18, -6), (dict(X=2 ** 26), 16, 16, -3),
])
def test_grouped_linear_refusals(moe, change, x_rows, offsets, code):
    d = moe.MoeLinearDims(**{**LIN, **change})
    assert moe._lib.moe_grouped_linear_f8(C.byref(d), 16, 16, x_rows, offsets, 16, 16, 16, None) == code


def _weights(moe, change=None, shared=True):
    w = {n: 16 for n, _ in moe.MoeWeightsF8._fields_ if shared or not n.startswith("sh_")}
    w.update(change or {})
    return moe.MoeWeightsF8(**w)


def _io(moe, **change):
    return moe.MoeNormIo(**{**dict(h=16, ldh=64, h_out=16, ldh_out=64), **change})


def test_layer_entry_points_refuse_before_launch(moe):
    lib = moe._lib
    d = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
    dsh = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8, n_shared=1, I_shared=64)
    norm = moe.MoeNorm(64, 16, 16, 1.0, 1e-6, 0.0)

    def ffn(dd, w, x_perm=16, off=16, x=16, y=16, ysh=16, ws=256, n=1 << 20):
        return lib.moe_expert_ffn_f8(C.byref(dd), x_perm, off, C.byref(w), x, y, ysh, ws, n, None)

    def fwd(dd, w, src=16, counts=16, local=None, ws=256, n=1 << 20, x=16, xq=None, xs=None, out=16, nm=None, io=None):
        ref = lambda v: None if v is None else C.byref(v)  # noqa: E731
        return lib.moe_forward_f8(C.byref(dd), None, 16, src, x, xq, xs, local, C.byref(w), counts, out, ref(nm), ref(io), None, ws, n, None)
    for name, _ in moe.MoeWeightsF8._fields_:
        for call in (ffn, fwd):
            assert call(dsh, _weights(moe, {name: None})) == moe.MOE_ERR_NULL, name
            bad = 18 if name.removeprefix("sh_").startswith("s_") else 24   # scales to 4 bytes, matrices to 16
            assert call(dsh, _weights(moe, {name: bad})) == moe.MOE_ERR_ALIGN, name
        if name.startswith("sh_"):   # not looked at without shared experts: the next check refuses
            assert ffn(d, _weights(moe, {name: None}), n=0) == moe.MOE_ERR_WORKSPACE
    w = _weights(moe)
    assert lib.moe_expert_ffn_f8(C.byref(d), 16, 16, None, 16, 16, 16, 256, 1 << 20, None) == moe.MOE_ERR_NULL
    assert ffn(d, w, x_perm=None) == moe.MOE_ERR_NULL and ffn(d, w, off=None) == moe.MOE_ERR_NULL
    assert ffn(d, w, y=None) == moe.MOE_ERR_NULL and ffn(dsh, w, x=None) == moe.MOE_ERR_NULL
    assert ffn(dsh, w, ysh=None) == moe.MOE_ERR_NULL and ffn(d, w, x_perm=24) == moe.MOE_ERR_ALIGN
    assert ffn(dsh, w, x=24) == moe.MOE_ERR_ALIGN and ffn(d, w, ws=None) == moe.MOE_ERR_WORKSPACE
    assert ffn(d, w, ws=128) == moe.MOE_ERR_ALIGN
    assert fwd(d, w, src=None) == moe.MOE_ERR_NULL and fwd(d, w, x=24) == moe.MOE_ERR_ALIGN
    assert fwd(moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=4), w) == moe.MOE_ERR_DIMS   # no placement list
    # the rows in one form, the output or an end
    assert fwd(d, w, x=None) == moe.MOE_ERR_NULL and fwd(d, w, x=None, xq=16) == moe.MOE_ERR_NULL
    assert fwd(d, w, xq=16, xs=16) == moe.MOE_ERR_DIMS and fwd(d, w, xs=16) == moe.MOE_ERR_NULL
    assert fwd(d, w, x=None, xq=24, xs=16) == moe.MOE_ERR_ALIGN and fwd(d, w, x=None, xq=16, xs=18) == moe.MOE_ERR_ALIGN
    assert fwd(d, w, x=None, xq=16, xs=16, n=0) == moe.MOE_ERR_WORKSPACE
    assert fwd(d, w, out=None) == moe.MOE_ERR_NULL and fwd(d, w, nm=norm) == moe.MOE_ERR_NULL
    assert fwd(d, w, io=_io(moe)) == moe.MOE_ERR_NULL and fwd(d, w, nm=norm, io=_io(moe), out=24) == moe.MOE_ERR_ALIGN
    assert fwd(d, w, nm=norm, io=_io(moe), out=None, n=0) == moe.MOE_ERR_WORKSPACE
    assert fwd(d, w, nm=moe.MoeNorm(56, 16, 16, 1.0, 1e-6, 0.0), io=_io(moe)) == moe.MOE_ERR_DIMS
    assert fwd(d, w, nm=norm, io=_io(moe, h=17)) == moe.MOE_ERR_ALIGN
    assert fwd(d, w, nm=norm, io=_io(moe, h_out=None)) == moe.MOE_ERR_NULL
    for call, entry in ((ffn, moe.ENTRY_EXPERT_FFN_F8), (fwd, moe.ENTRY_FORWARD_F8)):
        for dd in (d, dsh):
            need = moe.workspace_bytes(dd, entry)
            assert call(dd, w, n=need - 1) == moe.MOE_ERR_WORKSPACE
    for change in (dict(H=2 ** 17), dict(I=2 ** 17), dict(n_shared=2, I_shared=2 ** 16)):
        base = dict(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
        big = moe.dims(**{**base, **change})
        assert ffn(big, w) == moe.MOE_ERR_UNSUPPORTED and fwd(big, w) == moe.MOE_ERR_UNSUPPORTED
        for entry in (moe.ENTRY_EXPERT_FFN_F8, moe.ENTRY_FORWARD_F8):
            assert moe.workspace_bytes(big, entry) == 0
            assert moe.validate(big, entry, 1 << 62) == moe.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("change,T,code", [
    (dict(), -1, -2), (dict(ldh=63), 4, -2), (dict(ldh_out=63), 4, -2), (dict(x=16, ldx=63), 4, -2), (dict(q=16, scale=16, ldq=48), 4, -2),
    (dict(q=16, scale=16, ldq=72), 4, -6), (dict(q=16, ldq=64), 4, -1), (dict(scale=16), 4, -1), (dict(q=24, scale=16, ldq=64), 4, -6),
    (dict(q=16, scale=18, ldq=64), 4, -6), (dict(h=None), 4, -1), (dict(h=17), 4, -6), (dict(h_out=17), 4, -6), (dict(h_out=None), 4, -1),
    (dict(x=17, ldx=64), 4, -6), (dict(gate=16, gate_row=-1), 4, -2), (dict(gate=16, gate_col=2), 4, -2),
    (dict(gate=16, gate_row=63, gate_col=1), 4, -2), (dict(gate=17), 4, -6), (dict(ldh=2 ** 41), 4, -3),
    (dict(gate=16, gate_row=2 ** 41), 4, -3), (dict(h=None), 0, 0),
    (dict(ldh_out=72), 4, -2), (dict(ldh=72), 2, -2), (dict(h_out=32, x=16, ldx=72), 4, -2),  # in place, but rows over other rows
])
def test_norm_refusals(moe, change, T, code):
    n = moe.MoeNorm(64, 16, None, 1.0, 1e-6, 0.0)
    assert moe._lib.moe_norm_rows(C.byref(n), C.byref(_io(moe, **change)), T, 16, 64, None) == code


@pytest.mark.parametrize("T,rows,most,blocks", [
    (1, 4, 2 ** 20, 1), (4, 4, 2 ** 20, 1), (5, 4, 2 ** 20, 2), (5, 1, 2 ** 20, 5), (2 ** 22 - 1, 4, 2 ** 20, 2 ** 20), (7, 1, 3, 3),
    (2 ** 31 - 4, 4, 2 ** 20, 2 ** 20), (2 ** 31 - 3, 4, 2 ** 20, 2 ** 20), (2 ** 31 - 1, 4, 2 ** 20, 2 ** 20), (2 ** 31 - 1, 1, 2 ** 20, 2 ** 20),
    (2 ** 31 - 1, 4, 2 ** 31 - 1, 2 ** 29)])
def test_norm_workgroups(moe, T, rows, most, blocks):
    """Up to the most rows that 31 bits hold."""
    assert moe._lib.moe_test_norm_blocks(T, rows, most) == blocks


def test_norm_parameter_refusals(moe):
    f, ok = moe._lib.moe_norm_rows, moe.MoeNorm(64, 16, 16, 1.0, 1e-6, 0.0)
    io = _io(moe)
    assert f(None, C.byref(io), 4, 16, 64, None) == moe.MOE_ERR_NULL and f(C.byref(ok), None, 4, 16, 64, None) == moe.MOE_ERR_NULL
    assert f(C.byref(ok), C.byref(io), 4, 16, 63, None) == moe.MOE_ERR_DIMS and f(C.byref(ok), C.byref(io), 4, 17, 64, None) == moe.MOE_ERR_ALIGN
    assert f(C.byref(ok), C.byref(io), 4, 16, 2 ** 41, None) == moe.MOE_ERR_UNSUPPORTED
    for n, code in ((moe.MoeNorm(0, 16, 16, 1.0, 1e-6, 0.0), moe.MOE_ERR_DIMS), (moe.MoeNorm(64, 17, None, 1.0, 1e-6, 0.0), moe.MOE_ERR_ALIGN),
                    (moe.MoeNorm(64, None, 17, 1.0, 1e-6, 0.0), moe.MOE_ERR_ALIGN)):
        assert f(C.byref(n), C.byref(io), 4, 16, 64, None) == code
    wide = moe.MoeNorm(32769, None, None, 1.0, 1e-6, 0.0)
    assert f(C.byref(wide), C.byref(_io(moe, ldh=2 ** 16, ldh_out=2 ** 16)), 4, None, 0, None) == moe.MOE_ERR_UNSUPPORTED


def test_large_batches_gather_limit(moe):
    """forward_f8 reads token rows through 32-bit offsets, as forward_i8."""
    base = dict(H=7168, E=256, k=1, I=2048, S=1, E_local=32)
    assert moe.validate(moe.dims(T=299_000, **base), moe.ENTRY_FORWARD_F8, 1 << 62) == moe.MOE_OK
    assert moe.validate(moe.dims(T=300_000, **base), moe.ENTRY_FORWARD_F8, 1 << 62) == moe.MOE_ERR_UNSUPPORTED
    assert moe.validate(moe.dims(T=300_000, **base), moe.ENTRY_EXPERT_FFN_F8, 1 << 62) == moe.MOE_OK


@pytest.mark.parametrize("name", W.CONFIG_ORDER)
def test_workspaces_of_the_workloads(moe, name):
    cfg = W.CONFIGS[name]
    d = moe.dims_of(cfg)
    rows = cfg.T * cfg.k
    for entry in (moe.ENTRY_EXPERT_FFN_F8, moe.ENTRY_FORWARD_F8):
        need = moe.workspace_bytes(d, entry)
        assert need % 256 == 0
        assert moe.validate(d, entry, need) == moe.MOE_OK
        assert moe.validate(d, entry, need - 1) == moe.MOE_ERR_WORKSPACE
    # hidden rows in bf16 and in e4m3, the input rows in e4m3, a scale per 128 of either
    scales = 4 * -(-cfg.I // 128)
    assert moe.workspace_bytes(d, moe.ENTRY_EXPERT_FFN_F8) >= rows * (3 * cfg.I + scales + cfg.H)
    assert moe.workspace_bytes(d, moe.ENTRY_FORWARD_F8) >= rows * (3 * cfg.I + scales + 2 * cfg.H) + cfg.T * cfg.H


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=torch.uint8).view(F8) if dtype == F8 else torch.zeros(shape, dtype=dtype)


def test_binding_refuses_host_tensors_and_shapes(moe):
    x = zeros(4, 40)
    for f in (moe.quantize_rows_f8, moe.quantize_blocks_f8):
        with pytest.raises(ValueError, match="GPU"):
            f(x)
        with pytest.raises(TypeError):
            f(x.float())
        with pytest.raises(ValueError, match="contiguous"):
            f(x.t())
    with pytest.raises(ValueError, match="one behind the other"):
        moe.quantize_blocks_f8(zeros(2, 8, 40)[:, :4])
    q, s, w, ws, y = zeros(4, 48, dtype=F8), torch.zeros(4, 1), zeros(8, 48, dtype=F8), torch.zeros(1, 1), zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        moe.linear_f8(40, q, s, w, ws, y)
    with pytest.raises(TypeError):
        moe.linear_f8(40, q.view(torch.int8), s, w, ws, y)
    with pytest.raises(ValueError, match="at least 48"):
        moe.linear_f8(40, q[:, :40], s, w, ws, y)
    with pytest.raises(ValueError, match="rows of xq"):
        moe.linear_f8(40, q[:3], s, w, ws, y)
    with pytest.raises(ValueError, match="groups"):
        moe.grouped_linear_f8(40, q, s, None, w, ws, y)
    with pytest.raises(ValueError, match="one behind the other"):
        moe.grouped_linear_f8(40, q, s, None, zeros(2, 16, 48, dtype=F8)[:, :8], ws, y)
    d = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
    with pytest.raises(ValueError, match="w_gate"):
        moe.make_weights_f8(d, {})


def test_binding_refuses_rows_of_norms(moe):
    h = zeros(4, 40)
    with pytest.raises(ValueError, match="both or none"):
        moe.norm_io(h, q=zeros(4, 48, dtype=F8))
    with pytest.raises(ValueError, match="expected"):
        moe.norm_io(h, zeros(3, 40))
    with pytest.raises(ValueError, match="expected"):
        moe.norm_io(h, x=zeros(4, 41))
    with pytest.raises(ValueError, match="overlap"):
        moe.norm_io(zeros(1, 40).expand(4, 40))
    with pytest.raises(ValueError, match="contiguous"):
        moe.norm_io(zeros(40, 4).t())
    with pytest.raises(TypeError):
        moe.norm_io(h.float())
    with pytest.raises(ValueError, match="gate"):
        moe.norm_io(h, h, gate=zeros(2, 40))
    with pytest.raises(ValueError, match="gate"):
        moe.norm_io(h, h, gate=zeros(40))
    with pytest.raises(ValueError, match="gate"):
        moe.norm_io(h, h, gate=zeros(40, 4).t())
    with pytest.raises(TypeError):
        moe.norm_io(h, h, gate=zeros(4, 40).float())
    n, io = moe.norm(40), moe.norm_io(h, h)
    with pytest.raises(ValueError, match="GPU"):
        moe.norm_rows(n, io)
    with pytest.raises(ValueError, match="columns"):
        moe.norm_rows(moe.norm(48), io)
    with pytest.raises(ValueError, match="expected"):
        moe.norm_rows(n, io, y=zeros(5, 40))
    with pytest.raises(ValueError, match="GPU"):
        moe.norm(40, weight=zeros(40))


def test_binding_refuses_rows_of_the_layer(moe):
    d = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
    x, xq, xs = zeros(4, 64), zeros(4, 64, dtype=F8), torch.zeros(4, 1)
    n, io = moe.norm(64), moe.norm_io(x, x)
    call = lambda **kw: moe.forward_f8(d, None, None, kw.pop("x", None), None, {}, None, None, None, **kw)  # noqa: E731
    for kw in (dict(), dict(x=x, xq=xq, x_scale=xs), dict(xq=xq), dict(x=x, x_scale=xs)):
        with pytest.raises(ValueError, match="rows to the layer"):
            call(**kw)
    for kw in (dict(norm=n), dict(rows=io)):
        with pytest.raises(ValueError, match="both or none"):
            call(x=x, **kw)


def test_binding_refuses_sizes_of_31_bits(moe):
    """Sizes that the C interface would cut to 32 bits."""
    wide = torch.empty((1, 1), dtype=torch.bfloat16).expand(2 ** 31, 1)
    for f in (moe.quantize_rows_f8, moe.norm_io):
        with pytest.raises(moe.MoeError) as e:
            f(wide)
        assert e.value.status == moe.MOE_ERR_UNSUPPORTED


# ------------------------------------------------ which kernel a layer takes ----


ITEMS, TILES = 0, 1


def ffn_plan(moe, conf, T, quantised=0):
    out = (C.c_int64 * 8)()
    assert moe._lib.moe_test_ffn_f8_plan(C.byref(moe.dims(T=T, S=1, **conf)), quantised, out) == 0
    return out[0], out[4]


SHARE = dict(H=7168, E=256, k=8, I=2048, E_local=32)
LITE = dict(H=2048, E=64, k=6, I=1408, E_local=64, n_shared=2, I_shared=1408)
WIDE = dict(H=7168, E=256, k=1, I=2048, E_local=8, n_shared=1, I_shared=8192)


@pytest.mark.parametrize("conf,T,up,down", [
    # routed rows alone: their mean, 85
    (SHARE, 2719, ITEMS, ITEMS), (SHARE, 2720, TILES, TILES),
    # a shared expert beside them: half of the rows are in one matrix of 33
    (dict(SHARE, n_shared=1, I_shared=2048), 1000, ITEMS, ITEMS), (dict(SHARE, n_shared=1, I_shared=2048), 1500, TILES, TILES),
    (dict(SHARE, n_shared=1, I_shared=2048), 2700, TILES, TILES), (dict(SHARE, n_shared=1, I_shared=2048), 3300, TILES, TILES),
    # almost all of the work is shared
    (WIDE, 200, ITEMS, ITEMS), (WIDE, 1000, TILES, TILES), (WIDE, 8000, TILES, TILES),
    (dict(H=2048, E=64, k=4, I=1024, E_local=8, n_shared=1, I_shared=4096), 800, TILES, TILES),
    # a quarter is; the shared experts' K is not short
    (LITE, 400, ITEMS, ITEMS), (LITE, 600, ITEMS, ITEMS), (LITE, 900, TILES, TILES),
    # (short K of both)
    (dict(LITE, n_shared=1), 600, ITEMS, TILES),
])
def test_shared_rows_count_in_the_choice_of_kernel(moe, conf, T, up, down):
    for quantised in (0, 1):
        assert ffn_plan(moe, conf, T, quantised) == (up, down)


@pytest.mark.parametrize("M,N,K,G,pair", [
    # from the longer ring, a workgroup per CU, to the shorter one, two of them: 256 items of 64 weight rows
    (60, 12003, 4100, 0, 0), (777, 1003, 517, 0, 0), (16000, 60, 500, 0, 0), (256, 4096, 4096, 0, 0), (256, 4097, 4096, 0, 1),
    (150, 6001, 1300, 0, 1), (193, 7300, 641, 0, 1), (400, 4100, 700, 0, 1), (64, 16384, 4096, 0, 0), (64, 16385, 4096, 0, 0),
    (78, 3000, 700, 4, 0), (720, 1500, 1100, 12, 1), (1800, 700, 1500, 9, 1), (2500, 2100, 1700, 0, 0), (8, 517, 1003, 0, 0)])
def test_pairs_of_items_on_a_cu(moe, M, N, K, G, pair):
    d, out = moe.MoeLinearDims(M=M, N=N, K=K, G=G), C.c_int64(-1)
    assert moe._lib.moe_test_linear_f8_pair(C.byref(d), int(G > 0), C.byref(out)) == 0 and out.value == pair


def ffn_pairs(moe, conf, quantised=0):
    out = (C.c_int64 * 2)(-1, -1)
    assert moe._lib.moe_test_ffn_f8_pair(C.byref(moe.dims(S=1, **conf)), quantised, out) == 0
    return tuple(out)


def test_pairs_of_the_experts(moe):
    """Both sides are among the layers that the GPU tests hold against 64 bits."""
    pairs = {conf["T"]: ffn_pairs(moe, conf) for conf, up, down in FFN_KERNELS if (ITEMS, 2, 64) in (up, down)}
    assert pairs == {3000: (0, 1), 60: (0, 0), 300: (0, 0), 150: (0, 0), 400: (1, 1)}


# Parts of K of the products that quantise up to 8 tokens' rows (none: items), of
# gate/up and down, by tokens.
FEW_PARTS = [{1: (4, 4), 8: (4, 4)}, {1: (4, 4), 2: (2, 2), 3: (2, 2), 5: (1, 1), 8: (1, 1)}, {1: (2, 4), 2: (1, 4), 8: (1, 4)},
             {1: (4, 4), 8: (4, 4)}, {1: (1, 4), 3: (1, 4), 5: (1, None), 8: (1, None)}, {1: (1, 1), 5: (1, 1), 8: (None, 1)},
             {1: (4, 2), 2: (4, 1), 3: (4, 1), 5: (None, 1), 8: (None, 1)}]


@pytest.mark.parametrize("case", range(len(FEW)))
def test_parts_of_few_tokens(moe, case):
    """The layers of few tokens that the GPU tests run reach every cut."""
    assert len(FEW) == len(FEW_PARTS)
    for T, want in FEW_PARTS[case].items():
        out = (C.c_int64 * 8)()
        assert moe._lib.moe_test_ffn_f8_plan(C.byref(moe.dims(T=T, S=1, **FEW[case])), 0, out) == 0
        assert tuple(out[i + 1] if out[i] == 2 else None for i in (0, 4)) == want, T
    assert ffn_plan(moe, FEW[case], 9)[0] == ITEMS
