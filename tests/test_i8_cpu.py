"""The 8-bit entry points without a GPU: what they refuse, in which order and
with which code, the workspaces they ask for, and the binding's own checks."""
import ctypes as C

import pytest
import torch

from paper_2606_15177_amd import workloads as W


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
def test_quantize_rows_refusals(moe, rows, cols, x, ldx, q, ldq, scale, code):
    assert moe._lib.moe_quantize_rows(rows, cols, x, ldx, q, ldq, scale, None) == code


LIN = dict(M=4, N=8, K=40, G=2, X=4, ldx=48, ldw=48, ldy=8)


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), -2), (dict(N=0), -2), (dict(K=0), -2), (dict(ldx=32), -2), (dict(ldw=32), -2), (dict(ldy=7), -2),
    (dict(ldx=56), -6), (dict(ldw=56), -6), (dict(K=2 ** 17, ldx=2 ** 17, ldw=2 ** 17), -3), (dict(ldx=2 ** 21 + 16), -3),
    (dict(ldw=2 ** 21 + 16), -3), (dict(ldy=2 ** 21 + 1), -3), (dict(N=2 ** 24 + 1, ldy=2 ** 25), -3), (dict(M=0), 0),
])
def test_linear_refusals(moe, change, code):
    d = moe.MoeLinearDims(**{**LIN, **change})
    assert moe._lib.moe_linear_i8(C.byref(d), 16, 16, 16, 16, 16 if code else None, None) == code
    assert moe._lib.moe_grouped_linear_i8(C.byref(d), 16, 16, None, 16, 16, 16, 16 if code else None, None) == code


@pytest.mark.parametrize("ptrs,code", [
    ((None, 16, 16, 16, 16), -1), ((16, None, 16, 16, 16), -1), ((16, 16, None, 16, 16), -1), ((16, 16, 16, None, 16), -1),
    ((16, 16, 16, 16, None), -1), ((24, 16, 16, 16, 16), -6), ((16, 18, 16, 16, 16), -6), ((16, 16, 24, 16, 16), -6),
    ((16, 16, 16, 18, 16), -6), ((16, 16, 16, 16, 17), -6),
])
def test_linear_pointers(moe, ptrs, code):
    d = moe.MoeLinearDims(**LIN)
    xq, xs, wq, ws, y = ptrs
    assert moe._lib.moe_linear_i8(C.byref(d), xq, xs, wq, ws, y, None) == code
    assert moe._lib.moe_grouped_linear_i8(C.byref(d), xq, xs, None, 16, wq, ws, y, None) == code
    assert moe._lib.moe_linear_i8(None, xq, xs, wq, ws, y, None) == moe.MOE_ERR_NULL


@pytest.mark.parametrize("change,x_rows,offsets,code", [
    (dict(G=0), None, 16, -2), (dict(G=1025), None, 16, -3), (dict(X=-1), 16, 16, -2), (dict(), None, None, -1),
    (dict(), 18, 16, -6), (dict(), 16, 18, -6), (dict(X=2 ** 26), 16, 16, -3),
])
def test_grouped_linear_refusals(moe, change, x_rows, offsets, code):
    d = moe.MoeLinearDims(**{**LIN, **change})
    assert moe._lib.moe_grouped_linear_i8(C.byref(d), 16, 16, x_rows, offsets, 16, 16, 16, None) == code


def _i8_weights(moe, change=None, shared=True):
    w = {n: 16 for n, _ in moe.MoeWeightsI8._fields_ if shared or not n.startswith("sh_")}
    w.update(change or {})
    return moe.MoeWeightsI8(**w)


def test_layer_entry_points_refuse_before_launch(moe):
    lib = moe._lib
    d = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
    dsh = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8, n_shared=1, I_shared=64)
    ffn = lambda dd, w, x_perm=16, off=16, x=16, y=16, ysh=16, ws=256, n=1 << 20: lib.moe_expert_ffn_i8(  # noqa: E731
        C.byref(dd), x_perm, off, C.byref(w), x, y, ysh, ws, n, None)
    fwd = lambda dd, w, src=16, counts=16, local=None, ws=256, n=1 << 20, x=16: lib.moe_forward_i8(  # noqa: E731
        C.byref(dd), None, 16, src, x, local, C.byref(w), counts, 16, None, ws, n, None)
    for name, _ in moe.MoeWeightsI8._fields_:
        shared = name.startswith("sh_")
        for call in (ffn, fwd):
            assert call(dsh, _i8_weights(moe, {name: None})) == moe.MOE_ERR_NULL, name
            bad = 18 if name.removeprefix("sh_").startswith("s_") else 24   # scales to 4 bytes, matrices to 16
            assert call(dsh, _i8_weights(moe, {name: bad})) == moe.MOE_ERR_ALIGN, name
        if shared:   # not looked at without shared experts: the next check refuses
            assert ffn(d, _i8_weights(moe, {name: None}), n=0) == moe.MOE_ERR_WORKSPACE
    w = _i8_weights(moe)
    assert lib.moe_expert_ffn_i8(C.byref(d), 16, 16, None, 16, 16, 16, 256, 1 << 20, None) == moe.MOE_ERR_NULL
    assert ffn(d, w, x_perm=None) == moe.MOE_ERR_NULL and ffn(d, w, off=None) == moe.MOE_ERR_NULL
    assert ffn(d, w, y=None) == moe.MOE_ERR_NULL and ffn(dsh, w, x=None) == moe.MOE_ERR_NULL
    assert ffn(dsh, w, ysh=None) == moe.MOE_ERR_NULL and ffn(d, w, x_perm=24) == moe.MOE_ERR_ALIGN
    assert ffn(dsh, w, x=24) == moe.MOE_ERR_ALIGN and ffn(d, w, ws=None) == moe.MOE_ERR_WORKSPACE
    assert ffn(d, w, ws=128) == moe.MOE_ERR_ALIGN
    assert fwd(d, w, src=None) == moe.MOE_ERR_NULL and fwd(d, w, x=24) == moe.MOE_ERR_ALIGN
    assert fwd(moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=4), w) == moe.MOE_ERR_DIMS   # no placement list
    for call, entry in ((ffn, moe.ENTRY_EXPERT_FFN_I8), (fwd, moe.ENTRY_FORWARD_I8)):
        for dd in (d, dsh):
            need = moe.workspace_bytes(dd, entry)
            assert call(dd, w, n=need - 1) == moe.MOE_ERR_WORKSPACE
    # inner dimensions whose sums could pass int32
    for change in (dict(H=2 ** 17), dict(I=2 ** 17), dict(n_shared=2, I_shared=2 ** 16)):
        base = dict(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
        big = moe.dims(**{**base, **change})
        assert ffn(big, w) == moe.MOE_ERR_UNSUPPORTED and fwd(big, w) == moe.MOE_ERR_UNSUPPORTED
        for entry in (moe.ENTRY_EXPERT_FFN_I8, moe.ENTRY_FORWARD_I8):
            assert moe.workspace_bytes(big, entry) == 0
            assert moe.validate(big, entry, 1 << 62) == moe.MOE_ERR_UNSUPPORTED


def test_large_batches_gather_limit(moe):
    """forward_i8 reads token rows through 32-bit offsets: twice as many as moe_forward."""
    base = dict(H=7168, E=256, k=1, I=2048, S=1, E_local=32)
    assert moe.validate(moe.dims(T=299_000, **base), moe.ENTRY_FORWARD_I8, 1 << 62) == moe.MOE_OK
    assert moe.validate(moe.dims(T=300_000, **base), moe.ENTRY_FORWARD_I8, 1 << 62) == moe.MOE_ERR_UNSUPPORTED
    assert moe.validate(moe.dims(T=300_000, **base), moe.ENTRY_EXPERT_FFN_I8, 1 << 62) == moe.MOE_OK


@pytest.mark.parametrize("name", W.CONFIG_ORDER)
def test_workspaces_of_the_workloads(moe, name):
    cfg = W.CONFIGS[name]
    d = moe.dims_of(cfg)
    rows = cfg.T * cfg.k
    for entry in (moe.ENTRY_EXPERT_FFN_I8, moe.ENTRY_FORWARD_I8):
        need = moe.workspace_bytes(d, entry)
        assert need % 256 == 0
        assert moe.validate(d, entry, need) == moe.MOE_OK
        assert moe.validate(d, entry, need - 1) == moe.MOE_ERR_WORKSPACE
    # hidden rows in bf16 and in int8, the input rows in int8
    assert moe.workspace_bytes(d, moe.ENTRY_EXPERT_FFN_I8) >= rows * (3 * cfg.I + cfg.H)
    # the layer quantises each token once
    assert moe.workspace_bytes(d, moe.ENTRY_FORWARD_I8) >= rows * (3 * cfg.I + 2 * cfg.H) + cfg.T * cfg.H


def test_binding_refuses_host_tensors_and_shapes(moe):
    x = torch.zeros(4, 40, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        moe.quantize_rows(x)
    with pytest.raises(TypeError):
        moe.quantize_rows(x.float())
    with pytest.raises(ValueError, match="contiguous"):
        moe.quantize_rows(x.t())
    q, s, w, y = (torch.zeros(*n, dtype=t) for n, t in (((4, 48), torch.int8), ((4,), torch.float32), ((8, 48), torch.int8),
                                                        ((4, 8), torch.bfloat16)))
    ws = torch.zeros(8)
    with pytest.raises(ValueError, match="GPU"):
        moe.linear_i8(40, q, s, w, ws, y)
    with pytest.raises(ValueError, match="at least 48"):
        moe.linear_i8(40, q[:, :40], s, w, ws, y)
    with pytest.raises(ValueError, match="rows of xq"):
        moe.linear_i8(40, q[:3], s, w, ws, y)
    with pytest.raises(ValueError, match="groups"):
        moe.grouped_linear_i8(40, q, s, None, w, ws, y)
    with pytest.raises(ValueError, match="one behind the other"):
        moe.grouped_linear_i8(40, q, s, None, torch.zeros(2, 16, 48, dtype=torch.int8)[:, :8], ws, y)
    d = moe.dims(T=4, H=64, E=8, k=2, I=64, S=2, E_local=8)
    with pytest.raises(ValueError, match="w_gate"):
        moe.make_weights_i8(d, {})


def test_binding_checks_devices(moe):
    """Tensors of two devices, or a stream of another device than theirs, are refused."""
    class T:
        def __init__(self, d):
            self.get_device = lambda: d

    class S:
        device = torch.device("cuda:1")
        cuda_stream = 7
    with pytest.raises(ValueError, match="different devices"):
        moe._on_device(S(), T(0), None, T(1))
    with pytest.raises(ValueError, match="stream of"):
        moe._on_device(S(), T(0))
    with pytest.raises(ValueError, match="GPU"):
        moe._on_device(None, T(-1))
    assert moe._on_device(S(), None, T(1), T(1)) == (1, 7)


def test_calls_run_on_the_tensors_device(moe, monkeypatch):
    """With another device current, the call is made with the tensors' one as current."""
    seen, current = [], [0]

    class On:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            current[0] = self.d

        def __exit__(self, *a):
            current[0] = 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", On)

    class Lib:
        def moe_linear_i8(self, *a):
            seen.append(current[0])
            return a[0]
    monkeypatch.setattr(moe, "_lib", Lib())
    moe._call(1, "moe_linear_i8", 0)
    moe._call(0, "moe_linear_i8", 0)
    assert seen == [1, 0] and current == [0]
    with pytest.raises(RuntimeError, match="moe_linear_i8"):
        monkeypatch.setattr(moe, "strerror", lambda s: "text")
        moe._call(1, "moe_linear_i8", -3)


def linear_plan(moe, M, N, K, G=0):
    """(kernel, parts of K, rows of a tile or chunk) of a product, and HALF
    where a wave takes 16 weight rows."""
    d, out = moe.MoeLinearDims(M=M, N=N, K=K, G=G), (C.c_int64 * 4)()
    assert moe._lib.moe_test_linear_i8_plan(C.byref(d), int(G > 0), out) == 0
    return tuple(out[:3]) + ((HALF,) if out[3] else ())


ITEMS, TILES, FEW, HALF = 0, 1, 2, "half"


@pytest.mark.parametrize("M,N,K,G,plan", [
    (1, 2048, 7168, 0, (ITEMS, 4, 8, HALF)), (8, 4096, 512, 0, (ITEMS, 4, 8, HALF)), (8, 4097, 512, 0, (ITEMS, 4, 8)),
    (32, 4096, 512, 0, (ITEMS, 4, 32, HALF)), (32, 4097, 512, 0, (ITEMS, 4, 64)), (64, 2048, 512, 0, (ITEMS, 4, 32, HALF)),
    (64, 2049, 512, 0, (ITEMS, 4, 32)), (3, 128, 512, 8, (ITEMS, 4, 8, HALF)), (8, 8192, 512, 0, (ITEMS, 4, 8)), (8, 8193, 512, 0, (ITEMS, 2, 8)),
    (8, 16385, 512, 0, (ITEMS, 1, 128)), (9, 8192, 512, 0, (ITEMS, 4, 64)), (33, 4096, 512, 0, (ITEMS, 4, 32)),
    (33, 4097, 512, 0, (ITEMS, 4, 64)), (64, 16384, 512, 0, (ITEMS, 2, 64)), (64, 16385, 512, 0, (ITEMS, 1, 128)),
    (64, 16385, 4096, 0, (ITEMS, 2, 64)), (64, 32769, 4096, 0, (TILES, 1, 256)),
    (2560, 2048, 1500, 0, (TILES, 1, 256)), (2560, 1792, 1500, 0, (ITEMS, 1, 128)), (2560, 2048, 1499, 0, (ITEMS, 1, 128)),
    (4096, 2048, 1499, 0, (TILES, 1, 256)), (16384, 4096, 384, 0, (ITEMS, 1, 128)), (16384, 4096, 385, 0, (TILES, 1, 256)),
    (8 * 75, 4096, 1500, 8, (TILES, 1, 256)), (8 * 74, 4096, 1500, 8, (ITEMS, 1, 128)), (8 * 75, 3840, 1500, 8, (ITEMS, 1, 128)),
    (8 * 300, 6400, 1499, 8, (TILES, 1, 256)), (8 * 300, 6144, 1499, 8, (ITEMS, 1, 128)),
    (64 * 300, 1024, 2048, 64, (TILES, 1, 256)), (64 * 299, 1024, 2048, 64, (ITEMS, 1, 128)), (64 * 75, 1024, 2049, 64, (TILES, 1, 256)),
])
def test_products_take_the_kernel_of_their_sizes(moe, M, N, K, G, plan):
    assert linear_plan(moe, M, N, K, G) == plan


@pytest.mark.parametrize("change,up,down", [
    (dict(T=1), (FEW, 2, 1), (FEW, 2, 1)), (dict(T=8), (FEW, 1, 8), (FEW, 1, 8)), (dict(T=9), (ITEMS, 1, 128), (ITEMS, 1, 128)),
    (dict(T=1, I=64), (FEW, 4, 1), (FEW, 2, 1)), (dict(T=1, H=512, I=512), (FEW, 4, 1), (FEW, 4, 1)),
    # rows past half a CU's LDS are quantised by a launch of their own
    (dict(T=4, H=7168), (FEW, 2, 4), (FEW, 1, 4)), (dict(T=8, H=8000), (ITEMS, 1, 128), (FEW, 1, 8)),
    (dict(T=4096, H=2304, E=32, E_local=32, I=1536), (TILES, 1, 256), (TILES, 1, 256)),
])
def test_layers_take_the_kernel_of_their_sizes(moe, change, up, down):
    d = moe.dims(**{**dict(T=1, S=1, H=2048, E=128, k=8, I=768, E_local=128), **change})
    out = (C.c_int64 * 8)()
    assert moe._lib.moe_test_ffn_i8_plan(C.byref(d), out) == 0
    assert (tuple(out[:3]), tuple(out[4:7])) == (up, down) and not (out[3] or out[7])


@pytest.mark.parametrize("change,code", [(dict(X=0), -2), (dict(X=-1), -2), (dict(X=0, M=0), 0), (dict(X=1, M=0), 0)])
def test_grouped_linear_needs_a_row_to_gather(moe, change, code):
    """x_rows' entries outside [0, X) are rows of zeros, but some row has to be there."""
    d = moe.MoeLinearDims(**{**LIN, **change})
    assert moe._lib.moe_grouped_linear_i8(C.byref(d), 16, 16, 16, 16, 16, 16, 16, None) == code
    if code == 0:
        assert moe._lib.moe_grouped_linear_i8(C.byref(d), None, None, 16, 16, None, None, None, None) == 0


@pytest.mark.parametrize("M", [2 ** 31 - 255, 2 ** 31 - 127, 2 ** 31 - 1])
def test_rows_at_the_end_of_32_bits(moe, M):
    """A last tile or chunk of rows would end past int32: refused as a size, not as a failed launch."""
    for change in (dict(), dict(K=400, ldx=400, ldw=400), dict(N=1, ldy=1, K=1, ldx=16, ldw=16)):
        d = moe.MoeLinearDims(**{**LIN, "M": M, **change})
        assert moe._lib.moe_linear_i8(C.byref(d), 16, 16, 16, 16, 16, None) == moe.MOE_ERR_UNSUPPORTED
        for x_rows in (None, 16):
            assert moe._lib.moe_grouped_linear_i8(C.byref(d), 16, 16, x_rows, 16, 16, 16, 16, None) == moe.MOE_ERR_UNSUPPORTED
    for k in (1, 8):
        d = moe.dims(T=-(-M // k), H=8, E=8, k=k, I=8, S=1, E_local=8, n_shared=1, I_shared=8)
        for entry in (moe.ENTRY_EXPERT_FFN_I8, moe.ENTRY_FORWARD_I8):
            assert moe.validate(d, entry, 1 << 62) == moe.MOE_ERR_UNSUPPORTED
            assert moe.workspace_bytes(d, entry) == 0


def test_binding_refuses_sizes_past_32_bits(moe):
    """Sizes that the C structs cannot hold are refused, not cut to their low 32 bits."""
    def rows(n, cols, dtype=torch.int8):   # (of one row's memory)
        return torch.zeros((1, cols), dtype=dtype).expand(n, cols)
    many = 2 ** 32 + 4
    q, y, s = rows(4, 48), rows(4, 8, torch.bfloat16), torch.zeros(8)
    w, x_rows = torch.zeros((2, 8, 48), dtype=torch.int8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: moe.quantize_rows(rows(many, 40, torch.bfloat16)),
                 lambda: moe.linear_i8(40, rows(many, 48), s, rows(8, 48), s, rows(many, 8, torch.bfloat16)),
                 lambda: moe.grouped_linear_i8(40, rows(many, 48), s, s, w, s, rows(many, 8, torch.bfloat16)),
                 lambda: moe.grouped_linear_i8(40, rows(many, 48), s, s, w, s, y, x_rows=x_rows),
                 lambda: moe.grouped_linear_i8(40, q, s, s, torch.zeros((1, 1, 48), dtype=torch.int8).expand(many, 8, 48), s, y)):
        with pytest.raises(moe.MoeError, match="limits") as e:
            call()
        assert e.value.status == moe.MOE_ERR_UNSUPPORTED


@pytest.fixture
def recorded(moe, monkeypatch):
    """The binding's calls on host tensors: the library's arguments are recorded, nothing is launched."""
    calls = []
    monkeypatch.setattr(moe, "_on_device", lambda stream, *t: (0, 0))
    monkeypatch.setattr(moe, "_ptr", lambda t, dtypes=None: None if t is None else t.data_ptr())
    monkeypatch.setattr(moe, "_call", lambda dev, where, *args: calls.append((where, args)))
    return calls


def _host_layer(moe, T, n_shared):
    """Dims, every tensor argument of the two layer entries at exactly its size, and int8 weights."""
    d = moe.dims(T=T, H=40, E=8, k=2, I=24, S=3, E_local=5, n_shared=n_shared, I_shared=16)
    bf = dict(dtype=torch.bfloat16)
    t = dict(x_perm=torch.zeros((T * 2, 40), **bf), offsets=torch.zeros(6, dtype=torch.int32), x=torch.zeros((T, 40), **bf),
             y_perm=torch.zeros((T * 2, 40), **bf), y_shared=torch.zeros((T, 40), **bf), logits=torch.zeros((T, 8)),
             src=torch.zeros(T, dtype=torch.int32), local_experts=torch.zeros(5, dtype=torch.int32),
             counts=torch.zeros((3, 8), dtype=torch.int64), out=torch.zeros((T, 40), **bf))
    return d, t


def _host_weights(moe, EL=5, H=40, I=24, width=0):
    p = lambda n: (n + 15) // 16 * 16   # noqa: E731
    q, s = dict(dtype=torch.int8), dict(dtype=torch.float32)
    w = dict(w_gate=torch.zeros((EL, I, p(H)), **q), w_up=torch.zeros((EL, I, p(H)), **q), w_down=torch.zeros((EL, H, p(I)), **q),
             s_gate=torch.zeros((EL, I), **s), s_up=torch.zeros((EL, I), **s), s_down=torch.zeros((EL, H), **s))
    if width:
        w.update(sh_gate=torch.zeros((width, p(H)), **q), sh_up=torch.zeros((width, p(H)), **q), sh_down=torch.zeros((H, p(width)), **q),
                 sh_s_gate=torch.zeros(width, **s), sh_s_up=torch.zeros(width, **s), sh_s_down=torch.zeros(H, **s))
    return w


FFN_ARGS = ("x_perm", "offsets", "x", "y_perm", "y_shared")
FORWARD_ARGS = ("logits", "src", "x", "local_experts", "counts", "out")


def _ffn_call(moe, d, t, weights):
    moe.expert_ffn_i8(d, t["x_perm"], t["offsets"], weights, t["x"], t["y_perm"], t["y_shared"], None)


def _forward_call(moe, d, t, weights):
    moe.forward_i8(d, t["logits"], t["src"], t["x"], t["local_experts"], weights, t["counts"], t["out"], None)


@pytest.mark.parametrize("T", [1, 7])
@pytest.mark.parametrize("call,names", [(_ffn_call, FFN_ARGS), (_forward_call, FORWARD_ARGS)])
def test_layer_binding_refuses_short_tensors(moe, recorded, T, call, names):
    """Every tensor that the library reads or writes is as long as it will be read or written."""
    d, t = _host_layer(moe, T, 1)
    w = moe.make_weights_i8(d, _host_weights(moe, width=16))
    call(moe, d, t, w)
    assert len(recorded) == 1
    for name in names:
        short = {**t, name: t[name].flatten()[:-1]}
        with pytest.raises(ValueError, match=name):
            call(moe, d, short, w)
    assert len(recorded) == 1
    # left out: the library decides
    for name in ("x", "y_shared", "src", "local_experts", "counts"):
        if name in names and not (name == "x" and call is _forward_call):
            call(moe, d, {**t, name: None}, w)
    # not looked at by the library: no size to keep to
    d, t = _host_layer(moe, T, 0)
    w = moe.make_weights_i8(d, _host_weights(moe))
    if call is _ffn_call:
        call(moe, d, {**t, "x": t["x"][:0], "y_shared": t["y_shared"][:0]}, w)
    else:
        call(moe, d, {**t, "counts": None, "src": t["src"][:0]}, w)


@pytest.mark.parametrize("call", [_ffn_call, _forward_call])
def test_layer_binding_refuses_weights_of_other_sizes(moe, recorded, call):
    """A handle of int8 weights knows the sizes that it was made for."""
    d, t = _host_layer(moe, 3, 1)
    for change in (dict(EL=4), dict(H=32), dict(H=48), dict(I=16), dict(I=32), dict(width=0), dict(width=8), dict(width=24)):
        sizes = {**dict(EL=5, H=40, I=24, width=16), **change}
        other = moe.dims(T=9, H=sizes["H"], E=8, k=2, I=sizes["I"], S=1, E_local=sizes["EL"], n_shared=int(sizes["width"] > 0),
                         I_shared=sizes["width"])
        w = moe.make_weights_i8(other, _host_weights(moe, **sizes))
        with pytest.raises(ValueError, match="other sizes"):
            call(moe, d, t, w)
    assert not recorded
    # another batch, one expert more than hosted, shared experts that the layer does not use, a struct filled by hand
    call(moe, d, t, moe.make_weights_i8(_host_layer(moe, 50, 1)[0], _host_weights(moe, width=16)))
    more = moe.dims(T=3, H=40, E=8, k=2, I=24, S=3, E_local=6, n_shared=1, I_shared=16)
    w = moe.make_weights_i8(more, _host_weights(moe, EL=6, width=16))
    call(moe, d, t, w)
    call(moe, _host_layer(moe, 3, 0)[0], t, w)
    by_hand = moe.MoeWeightsI8(**{n: 16 for n, _ in moe.MoeWeightsI8._fields_})
    call(moe, d, t, by_hand)
    assert len(recorded) == 4


@pytest.mark.parametrize("call", [_ffn_call, _forward_call])
def test_layer_binding_takes_a_dict_of_weights(moe, recorded, call):
    """As expert_ffn and forward do."""
    d, t = _host_layer(moe, 3, 1)
    tensors = _host_weights(moe, width=16)
    call(moe, d, t, tensors)
    call(moe, d, t, moe.make_weights_i8(d, tensors))
    seen = [next(a._obj for a in args if isinstance(getattr(a, "_obj", None), moe.MoeWeightsI8)) for _, args in recorded]
    assert all(getattr(seen[0], n) == tensors[n].data_ptr() == getattr(seen[1], n) for n in tensors)
    with pytest.raises(ValueError, match="w_down"):
        call(moe, d, t, {**tensors, "w_down": tensors["w_down"][:4]})
    with pytest.raises(TypeError, match="bf16"):
        call(moe, d, t, moe.MoeWeights())


@pytest.mark.parametrize("kind", ["none", "torch", "int", "pointer", "object", "null", "legacy"])
def test_outputs_belong_to_the_stream_they_are_written_on(moe, recorded, monkeypatch, kind):
    """What quantize_rows and MoeLayerI8.forward allocate is that stream's in
    torch's allocator, a raw handle's too: freed early, it is not handed out to
    the current stream while the launch may still write it."""
    entered = []

    class Stream:
        def __init__(self, name):
            self.name = name
            self.cuda_stream = 48

    class External(Stream):
        def __init__(self, handle, device):
            super().__init__(("external", handle, device))

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            entered.append(self.s and self.s.name)

        def __exit__(self, *a):
            pass
    for name, fake in (("Stream", Stream), ("ExternalStream", External), ("stream", On), ("default_stream", lambda dev: Stream(("default", dev)))):
        monkeypatch.setattr(torch.cuda, name, fake)

    class Handle:
        cuda_stream = 64
    stream, where = {"none": (None, None), "torch": (Stream("torch"), "torch"), "int": (48, ("external", 48, 0)),
                     "pointer": (C.c_void_p(48), ("external", 48, 0)), "object": (Handle(), ("external", 64, 0)),
                     "null": (C.c_void_p(None), ("default", 0)), "legacy": (1, ("default", 0))}[kind]
    x = torch.zeros((3, 40), dtype=torch.bfloat16)
    moe.quantize_rows(x, stream=stream)
    assert entered == [where]
    d, t = _host_layer(moe, 3, 0)
    layer = moe.MoeLayerI8(d, _host_weights(moe), t["local_experts"], device="cpu")
    layer.forward(t["logits"], None, t["x"], stream=stream)
    assert entered == [where, where] and [c[0] for c in recorded] == ["moe_quantize_rows", "moe_forward_i8"]
    # given ones are the caller's
    moe.quantize_rows(x, torch.zeros((3, 48), dtype=torch.int8), torch.zeros(3), stream=stream)
    layer.forward(t["logits"], None, t["x"], out=t["out"], stream=stream)
    assert len(entered) == 2


def test_one_row_has_no_stride(moe, recorded):
    """A single row may be cut from a longer one at any length: the stride that
    goes to the library is one that it takes, whatever the row's tensor says."""
    row = torch.zeros((1, 2 ** 21 + 100), dtype=torch.int8)
    bf, s = torch.zeros((1, 90), dtype=torch.bfloat16), torch.zeros(4)

    def dims():
        d = next(a._obj for a in recorded[-1][1] if hasattr(a, "_obj"))
        return d.ldx, d.ldw, d.ldy
    for cols in (48, 50, 63, 2 ** 21 + 100):
        moe.linear_i8(40, row[:, :cols], s, row[:, :cols], s, bf[:, :1])
        assert dims() == (48, 48, 1)
        moe.grouped_linear_i8(40, row[:, :cols], s, s, row[None, :, :cols], s, bf[:, :1])
        assert dims() == (48, 48, 1)
        moe.quantize_rows(bf[:, :40], row[:, :cols], s)
        assert recorded[-1][1][3] == 40 and recorded[-1][1][5] == 48
    # several rows: as they lie, odd distances for the library to refuse
    moe.linear_i8(40, torch.zeros((2, 50), dtype=torch.int8), s, torch.zeros((3, 80), dtype=torch.int8)[:, :48], s,
                  torch.zeros((2, 7), dtype=torch.bfloat16)[:, :3])
    assert dims() == (50, 80, 7)


@pytest.mark.parametrize("M,N,G,tiles,grid,parts", [
    (2500, 2100, 0, 90, 256, 2), (2560, 2048, 0, 80, 256, 2), (2048, 4096, 0, 128, 256, 2), (2048, 4097, 0, 136, 256, 1),   # an only round
    (2048, 2048, 0, 64, 256, 4), (2048, 2049, 0, 72, 256, 2), (256, 256, 0, 1, 8, 4), (1280, 1024, 0, 20, 80, 4),
    (5003, 3801, 0, 300, 256, 4), (5003, 4400, 0, 360, 256, 2), (5003, 5000, 0, 400, 256, 1),                             # past one of 256
    (4096, 2048, 4, 48, 256, 4), (4096, 2048, 4, 96, 256, 2), (4096, 2048, 4, 160, 256, 1),                               # groups with few rows
])
def test_tiles_of_a_last_round_run_in_parts(moe, M, N, G, tiles, grid, parts):
    """(on 256 CUs)"""
    d, out = moe.MoeLinearDims(M=M, N=N, K=1700, G=G), (C.c_int64 * 2)()
    assert G or tiles == -(-M // 256) * -(-N // 256)
    assert moe._lib.moe_test_linear_i8_round(C.byref(d), int(G > 0), tiles, out) == 0
    assert tuple(out) == (grid, parts)


@pytest.mark.parametrize("M,N,K,G,R,plan,as_m", [
    (5120, 2048, 4096, 64, 1280, (ITEMS, 1, 128), (TILES, 1, 256)),     # a quarter of the experts hosted, 20 rows each
    (5120, 2048, 4096, 64, 64 * 75, (TILES, 1, 256), (TILES, 1, 256)), (5120, 2048, 4096, 64, 64 * 74, (ITEMS, 1, 128), (TILES, 1, 256)),
    (4096, 512, 1024, 64, 16, (ITEMS, 4, 64), (ITEMS, 1, 128)),         # most groups empty: fewer items than CUs
])
def test_grouped_products_take_the_kernel_of_their_expected_rows(moe, M, N, K, G, R, plan, as_m):
    """y may have room for more rows than there will be (M); R says how many."""
    for r, want in ((R, plan), (0, as_m), (M, as_m), (-1, as_m), (M + 1, as_m), (2 ** 31 - 1, as_m), (-2 ** 31, as_m)):
        d, out = moe.MoeLinearDims(M=M, N=N, K=K, G=G, R=r), (C.c_int64 * 4)()
        assert moe._lib.moe_test_linear_i8_plan(C.byref(d), 1, out) == 0
        assert tuple(out[:3]) == want and not out[3], r
    dense, out = moe.MoeLinearDims(M=M, N=N, K=K, G=G, R=R), (C.c_int64 * 4)()
    assert moe._lib.moe_test_linear_i8_plan(C.byref(dense), 0, out) == 0 and tuple(out[:3]) == linear_plan(moe, M, N, K)


def test_binding_passes_the_expected_rows(moe, recorded):
    y, w = torch.zeros((40, 8), dtype=torch.bfloat16), torch.zeros((2, 8, 48), dtype=torch.int8)
    q, s, o = torch.zeros((40, 48), dtype=torch.int8), torch.zeros(40), torch.zeros(3, dtype=torch.int32)
    for rows, r in ((None, 0), (7, 7), (0, 0)):
        moe.grouped_linear_i8(40, q, s, o, w, s, y, rows=rows)
        assert next(a._obj for a in recorded[-1][1] if hasattr(a, "_obj")).R == r


TAPS = ("topk_idx", "topk_w", "expert_load", "offsets", "perm_token", "inv_pos")


def test_forward_binding_checks_taps_and_bias(moe, recorded, monkeypatch):
    """Extra outputs and the gate's bias are as long as the layer takes them to
    be, live where it runs, and are kept as long as the structs that point at them."""
    d, t = _host_layer(moe, 7, 0)
    d.flags = moe.GATE_SIGMOID
    w = moe.make_weights_i8(d, _host_weights(moe))
    sizes = dict(topk_idx=14, topk_w=14, expert_load=8, offsets=6, perm_token=14, inv_pos=14)

    def call(taps=None, gating=None):
        moe.forward_i8(d, t["logits"], t["src"], t["x"], t["local_experts"], w, t["counts"], t["out"], None, taps=taps, gating=gating)
    for name in TAPS:
        dtype = torch.float32 if name == "topk_w" else torch.int32
        tensor = torch.zeros(sizes[name], dtype=dtype)
        call(moe.make_taps(**{name: tensor}))
        assert moe.make_taps(**{name: tensor}).tensors[name] is tensor
        with pytest.raises(ValueError, match=name):
            call(moe.make_taps(**{name: tensor[:-1]}))
    call(moe.make_taps(), moe.gating(torch.zeros(8)))
    with pytest.raises(ValueError, match="bias"):
        call(gating=moe.gating(torch.zeros(7)))
    call(moe.MoeTaps(), moe.MoeGating(None, 1.0, 0, 0))   # filled in by hand
    seen = []
    monkeypatch.setattr(moe, "_on_device", lambda stream, *tensors: (seen.extend(tensors), (0, 0))[1])
    bias, idx = torch.zeros(8), torch.zeros(14, dtype=torch.int32)
    call(moe.make_taps(topk_idx=idx), moe.gating(bias))
    assert any(s is bias for s in seen) and any(s is idx for s in seen)
