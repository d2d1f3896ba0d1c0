"""The e4m3 operators on the GPU against their definitions in 64 bits.

Quantisation: values and scales bit for bit.  Products and the experts' networks:
within the bounds that their arithmetic leaves (f8_util.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.f8_util import (BF16, F8, blocks, blocks_exactly, ffn_and_bound, gen, pad16, product_and_error, randn, rows_exactly,
                           to_f8)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    from paper_2606_15177_amd import moe
    return moe


# ---------------------------------------------------------------- quantise ----


def raw(t):
    return t.view(torch.uint8)


def assert_quantized(moe, x):
    rows, cols = x.shape
    kb = blocks(cols)
    q = torch.full((rows + 2, pad16(cols) + 32), 77, dtype=torch.uint8, device="cuda").view(F8)
    scale = torch.full((rows + 2, kb), 5.0, device="cuda")
    moe.quantize_rows_f8(x, q[1:rows + 1, 16:16 + pad16(cols)], scale[1:rows + 1])
    ref, ref_s = rows_exactly(x)
    got = q[1:rows + 1, 16:16 + cols]
    assert torch.equal(got.double(), ref)
    assert torch.equal(scale[1:rows + 1], ref_s)
    b = raw(q).clone()
    assert (b[1:rows + 1, 16 + cols:16 + pad16(cols)] == 0).all()        # the padding
    b[1:rows + 1, 16:16 + pad16(cols)] = 77
    assert (b == 77).all() and (scale[0] == 5.0).all() and (scale[rows + 1] == 5.0).all()  # and nothing else


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 16), (2, 127), (2, 128), (2, 129), (2, 517), (64, 2048), (9, 2049),
                                       (7, 4096), (3, 16384), (2, 20001), (1030, 264), (1, 7168), (300, 40)])
def test_quantize_rows(moe, rows, cols):
    assert_quantized(moe, randn((rows, cols), rows * 31 + cols))


@pytest.mark.parametrize("cols,stride,offset", [(100, 101, 0), (100, 133, 1), (37, 41, 3), (2050, 2051, 1), (8, 24, 5)])
def test_quantize_rows_strided_and_unaligned(moe, cols, stride, offset):
    flat = randn((6 * stride + 8,), cols)
    assert_quantized(moe, flat[offset:offset + 6 * stride].view(6, stride)[:, :cols])


def tie_rows():
    """Rows of 256 columns (two groups): every tie between e4m3 values, and every
    8-bit significand, against maxima that put ties on them exactly."""
    normal = [(8 + m + 0.5) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)]
    ties = [v for v in normal if v < 448.0] + [(m + 0.5) * 2.0 ** -9 for m in range(8)]
    sig = [s * 2.0 ** -k for s in range(128, 256) for k in (0, 5)]
    rows = []
    for a in (448.0, 224.0, 1.75, 3.5 * 2.0 ** 20, 1.0, 255.0, 129.0):
        for values in (ties, sig[::2], sig[1::2]):
            v = (np.array(values) * (a / 448.0 if values is ties else a / 512.0))[:125]
            for sign in (1.0, -1.0):
                g = np.zeros(256)
                g[:len(v)], g[127], g[128] = sign * v, a, -a
                rows.append(g)
    return torch.tensor(np.array(rows))


def test_quantize_rows_ties_and_extremes(moe):
    x = tie_rows().cuda()
    exact = x.to(torch.bfloat16).double() == x
    assert exact.double().mean() > 0.5    # (the ties are among them where the maximum is 7 times a power of two)
    x = x.to(torch.bfloat16)
    for scale in (1.0, 2.0 ** 100, 2.0 ** -100, 2.0 ** -126):   # up to fp32's ends
        assert_quantized(moe, (x.float() * scale).to(torch.bfloat16))
    tiny = torch.zeros((3, 40), dtype=torch.int16, device="cuda")
    tiny[0, :5] = torch.tensor([1, 2, 3, 127, -32767], dtype=torch.int16)   # subnormal bf16
    tiny[1, 7] = 1
    assert_quantized(moe, tiny.view(torch.bfloat16))
    big = torch.tensor([[3.3895313892515355e38, -1.0, 0.0, 2e38] * 5], device="cuda").to(torch.bfloat16)
    assert_quantized(moe, big)


@pytest.mark.parametrize("cols", [5, 2100])
def test_quantize_rows_not_finite(moe, cols):
    """NaN and infinities take the 128 columns that hold them, no others."""
    x = randn((5, cols), 9)
    x[0, 3], x[1, cols - 1], x[2, 0] = float("nan"), float("inf"), float("-inf")
    x[3] = 0.0
    q, s = moe.quantize_rows_f8(x)
    ref, ref_s = rows_exactly(torch.where(torch.isfinite(x), x, torch.zeros_like(x)))
    bad = torch.zeros((5, blocks(cols)), dtype=torch.bool, device="cuda")
    bad[0, 0], bad[1, -1], bad[2, 0] = True, True, True
    assert torch.isnan(s[bad]).all() and torch.equal(s[~bad], ref_s[~bad]) and (s[3] == 0).all()
    cut = torch.repeat_interleave(bad, 128, dim=1)[:, :cols]
    got = q[:, :cols].double()
    assert (got[cut] == 0).all() and torch.equal(got[~cut], ref[~cut])


def test_quantize_no_rows(moe):
    q, s = moe.quantize_rows_f8(torch.empty((0, 140), dtype=torch.bfloat16, device="cuda"))
    assert q.shape == (0, 144) and s.shape == (0, 2) and q.dtype == F8
    q, s = moe.quantize_blocks_f8(torch.empty((0, 3, 140), dtype=torch.bfloat16, device="cuda"))
    assert q.shape == (0, 3, 144) and s.shape == (0, 1, 2)


@pytest.mark.parametrize("G,rows,cols", [(1, 1, 1), (1, 128, 128), (2, 129, 127), (3, 257, 260), (5, 40, 1003), (1, 520, 1000), (40, 3, 9)])
def test_quantize_blocks(moe, G, rows, cols):
    x = randn((G, rows, cols), G + rows)
    q = torch.full((G, rows, pad16(cols)), 77, dtype=torch.uint8, device="cuda").view(F8)
    got_q, got_s = moe.quantize_blocks_f8(x, q)
    ref, ref_s = blocks_exactly(x)
    assert got_q is q and torch.equal(q[..., :cols].double(), ref) and torch.equal(got_s, ref_s)
    assert (raw(q)[..., cols:] == 0).all()
    one_q, one_s = moe.quantize_blocks_f8(x[-1])
    assert torch.equal(raw(one_q), raw(q[-1])) and torch.equal(one_s, got_s[-1])


def test_quantize_blocks_strided_and_not_finite(moe):
    wide = randn((2, 300, 419), 3)
    x = wide[..., 3:403]
    x[1, 290, 399] = float("nan")
    x[0, :128, 128:256] = 0.0
    qw = torch.full((2, 300, 448), 77, dtype=torch.uint8, device="cuda").view(F8)
    s = torch.empty((2, 3, 4), device="cuda")
    moe.quantize_blocks_f8(x, qw[..., 16:416], s)
    ref, ref_s = blocks_exactly(torch.where(torch.isfinite(x), x, torch.zeros_like(x)))
    bad = torch.zeros((2, 3, 4), dtype=torch.bool, device="cuda")
    bad[1, 2, 3] = True
    assert torch.isnan(s[bad]).all() and torch.equal(s[~bad], ref_s[~bad]) and s[0, 0, 1] == 0
    ref[1, 256:, 384:] = 0.0
    assert torch.equal(qw[..., 16:416].double(), ref)
    assert (raw(qw)[..., :16] == 77).all() and (raw(qw)[..., 416:] == 77).all()


# ---------------------------------------------------------------- products ----


def operands(M, N, K, seed, G=None):
    """Quantised in torch, so that a product's test does not rest on the quantiser."""
    q, xs = rows_exactly(randn((M, K), seed))
    w, ws = blocks_exactly(randn((G or 1, N, K), seed + 1, 0.02) * torch.linspace(0.5, 2.0, N, device="cuda").to(torch.bfloat16)[:, None])
    wq = to_f8(w)
    return to_f8(q), xs, (wq if G is not None else wq[0]), (ws if G is not None else ws[0])


def assert_product(y, xq, xs, wq, ws, K, rows=None):
    if rows is not None:
        xq, xs = xq.view(torch.uint8)[rows].view(F8), xs[rows]
    ref, _, err = product_and_error(xq, xs, wq, ws, K)
    off = (y.double() - ref).abs()
    bound = err + (ref.abs() + err) * BF16
    assert (off <= bound).all(), (off / bound).max().item()


SIZES = [(1, 1, 1), (1, 64, 16), (1, 2048, 7168), (3, 17, 33), (16, 300, 100), (31, 129, 640), (33, 1003, 517),
         (64, 512, 4096), (65, 256, 2048), (127, 384, 1000), (129, 96, 272), (200, 1000, 1408), (257, 520, 128),
         (513, 257, 4100), (777, 1003, 517), (1500, 640, 768), (40, 128, 14336), (2050, 1280, 384)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(moe, M, N, K):
    xq, xs, wq, ws = operands(M, N, K, M + N + K)
    y = torch.full((M + 1, N), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.linear_f8(K, xq, xs, wq, ws, y[:M])
    assert_product(y[:M], xq, xs, wq, ws, K)
    assert (y[M] == 3.0).all()


@pytest.mark.parametrize("M,N,K", [(5, 40, 50), (70, 200, 300), (300, 130, 1000), (600, 256, 64)])
def test_linear_strides(moe, M, N, K):
    """Rows of inputs, weights and results that lie apart (NaN between them),
    results at any bf16 address."""
    xq, xs, wq, ws = operands(M, N, K, M)
    xb = torch.full((M, pad16(K) + 32), 0x7f, dtype=torch.uint8, device="cuda").view(F8)
    wb = torch.full((N, pad16(K) + 64), 0x7f, dtype=torch.uint8, device="cuda").view(F8)
    raw(xb)[:, 16:16 + pad16(K)], raw(wb)[:, 32:32 + pad16(K)] = raw(xq), raw(wq)
    yb = torch.full((M, N + 13), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.linear_f8(K, xb[:, 16:16 + pad16(K)], xs, wb[:, 32:32 + pad16(K)], ws, yb[:, 5:5 + N])
    assert_product(yb[:, 5:5 + N], xq, xs, wq, ws, K)
    assert (yb[:, :5] == 3.0).all() and (yb[:, 5 + N:] == 3.0).all()


@pytest.mark.parametrize("M", [2, 300])
def test_linear_values(moe, M):
    """Every e4m3 value meets every other: products of single columns are exact
    but for the rounding to bf16."""
    bits = torch.arange(256, dtype=torch.uint8, device="cuda")
    bits = bits[(bits & 0x7f) != 0x7f]
    K = 16
    x, w = torch.zeros((M, K), dtype=torch.uint8, device="cuda"), torch.zeros((254, K), dtype=torch.uint8, device="cuda")
    w[:, 5] = bits
    for first in range(0, 254, M):
        part = bits[first:first + M]
        x[:, 5] = 0
        x[:len(part), 5] = part
        y = torch.empty((M, 254), dtype=torch.bfloat16, device="cuda")
        ones = torch.ones((max(M, 2), 1), device="cuda")
        moe.linear_f8(K, x.view(F8), ones[:M], w.view(F8), ones[:2], y)
        ref = (x.view(F8).double()[:, 5:6] @ w.view(F8).double()[:, 5:6].t()).to(torch.bfloat16)
        assert torch.equal(y, ref)


def test_linear_scales(moe):
    """Scales of any size and sign; zero, NaN and infinite ones; NaN operands."""
    M, N, K = 5, 300, 500
    xq, xs, wq, ws = operands(M, N, K, 3)
    xs, ws = xs * torch.tensor([2.0 ** 60, -1.0, 1.0, 0.0, 2.0 ** -70], device="cuda")[:, None], ws * -0.37
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    moe.linear_f8(K, xq, xs, wq, ws, y)
    assert_product(y, xq, xs, wq, ws, K)
    assert (y[3] == 0).all()
    xs[1, 2], ws[0, 1] = float("nan"), float("inf")
    raw(xq)[2, 7], raw(wq)[299, 3] = 0x7f, 0xff
    moe.linear_f8(K, xq, xs, wq, ws, y)
    nan = torch.isnan(y)
    assert nan[1].all() and nan[2].all() and nan[:, 299].all() and nan[3, :128].all() and not nan[[0, 4]][:, 128:299].any()
    assert torch.isinf(y[[0, 4], :128]).all()


def test_linear_no_rows(moe):
    _, _, wq, ws = operands(1, 8, 32, 0)
    e = torch.empty
    moe.linear_f8(32, e((0, 32), dtype=F8, device="cuda"), e((0, 1), device="cuda"), wq, ws, e((0, 8), dtype=torch.bfloat16, device="cuda"))


def grouped_case(sizes, N, K, seed, first=0, spare=3, gather=None):
    """Operands of groups of the given sizes; rows before the first group and
    behind the last one belong to none."""
    G, R = len(sizes), sum(sizes)
    M = first + R + spare
    xq, xs, wq, ws = operands(gather or M, N, K, seed, G)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]) + first, dtype=torch.int32, device="cuda")
    x_rows = None
    if gather:
        x_rows = torch.randint(0, gather, (M,), generator=gen(seed), device="cuda", dtype=torch.int32)
    return M, xq, xs, wq, ws, offsets, x_rows


def check_grouped(moe, sizes, N, K, seed, **kw):
    M, xq, xs, wq, ws, offsets, x_rows = grouped_case(sizes, N, K, seed, **kw)
    y = torch.full((M, N), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.grouped_linear_f8(K, xq, xs, offsets, wq, ws, y, x_rows=x_rows)
    o = offsets.tolist()
    for g in range(len(sizes)):
        if o[g] < o[g + 1]:
            rows = slice(o[g], o[g + 1]) if x_rows is None else x_rows[o[g]:o[g + 1]].long()
            assert_product(y[o[g]:o[g + 1]], xq, xs, wq[g], ws[g], K, rows)
    assert (y[:o[0]] == 3.0).all() and (y[o[-1]:] == 3.0).all()


def ragged(G, mean, seed, hot=0):
    rng = np.random.default_rng(seed)
    s = rng.poisson(mean, G) * (rng.random(G) < 0.8)
    if hot:
        s[rng.integers(G)] = hot
    return s.tolist()


GROUPS = [([0], 16, 16), ([1], 130, 48), ([0, 0, 5, 0], 64, 100), ([1] * 70, 200, 264), ([3, 0, 64, 65, 128, 129, 1], 300, 96),
          ([256, 255, 257, 0, 384, 511], 384, 640), (ragged(128, 16, 1), 768, 2048), (ragged(64, 60, 2, 700), 520, 1408),
          (ragged(300, 3, 3), 96, 80), (ragged(1024, 1, 4), 64, 48), ([2000, 1, 0, 900], 1003, 517),
          (ragged(9, 200, 5, 1300), 256, 4100), ([1000, 900, 1100, 800, 1200, 0, 300], 1024, 1024)]


@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_grouped_linear(moe, case):
    sizes, N, K = GROUPS[case]
    check_grouped(moe, sizes, N, K, case)


@pytest.mark.parametrize("case", range(len(GROUPS)))
def test_grouped_linear_gathered(moe, case):
    sizes, N, K = GROUPS[case]
    check_grouped(moe, sizes, N, K, case + 100, gather=max(1, sum(sizes) // 3), first=case % 3)


@pytest.mark.parametrize("sizes", [[5, 9, 0, 2], [300, 20, 0, 600]])
def test_grouped_linear_rows_out_of_range(moe, sizes):
    """Entries of x_rows outside x stand for rows of zeros, whatever scales there are."""
    N, K = 72, 112
    M, xq, xs, wq, ws, offsets, x_rows = grouped_case(sizes, N, K, 5, gather=11)
    xs[0] = float("nan")
    x_rows[x_rows == 0] = 1
    x_rows[0], x_rows[3], x_rows[sizes[0] + 1], x_rows[M - 4] = -1, 11, 2 ** 31 - 1, -2 ** 31
    y = torch.full((M, N), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.grouped_linear_f8(K, xq, xs, offsets, wq, ws, y, x_rows=x_rows)
    bad = ((x_rows < 0) | (x_rows >= 11))[:sum(sizes)]
    assert (y[:sum(sizes)][bad] == 0).all() and bad.sum() == 4
    ok = (~bad).nonzero().flatten()
    g = torch.repeat_interleave(torch.arange(4, device="cuda"), torch.tensor(sizes, device="cuda"))
    for e in range(4):
        r = ok[g[ok] == e]
        if len(r):
            assert_product(y[r], xq, xs, wq[e], ws[e], K, x_rows[r].long())


@pytest.mark.parametrize("offsets", [[-5, 3, 2, 900], [4, 4, 2 ** 31 - 1, -2 ** 31]])
def test_grouped_linear_offsets_out_of_range(moe, offsets):
    """Offsets that are none: no row outside y is touched, nothing ends."""
    N, K, M = 40, 260, 30
    _, xq, xs, wq, ws, _, _ = grouped_case([10, 10, 10], N, K, 5, spare=0)
    y = torch.full((M + 8, N), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.grouped_linear_f8(K, xq, xs, torch.tensor(offsets, dtype=torch.int32, device="cuda"), wq, ws, y[4:4 + M])
    torch.cuda.synchronize()
    assert (y[:4] == 3.0).all() and (y[4 + M:] == 3.0).all()


# ------------------------------------------------------ experts and layer ----


def layer_weights(moe, d, seed):
    def n(shape, k):
        return randn(shape, seed + k, 0.05)
    w = {"w_gate": n((d.E_local, d.I, d.H), 0), "w_up": n((d.E_local, d.I, d.H), 1), "w_down": n((d.E_local, d.H, d.I), 2)}
    if d.n_shared:
        w.update(sh_gate=n((d.n_shared, d.I_shared, d.H), 3), sh_up=n((d.n_shared, d.I_shared, d.H), 4),
                 sh_down=n((d.n_shared, d.H, d.I_shared), 5))
    return w, moe.quantize_weights_f8(d, w)


def test_quantize_weights(moe):
    """Layouts and blocks: the shared experts' down rows lie side by side."""
    d = moe.dims(4, 136, 6, 2, 264, 1, 3, 2, 72)
    w, q = layer_weights(moe, d, 7)
    for name in ("gate", "up", "down"):
        t = w["w_" + name]
        ref, ref_s = blocks_exactly(t)
        assert torch.equal(q["w_" + name][..., :t.shape[-1]].double(), ref) and torch.equal(q["s_" + name], ref_s)
    down = torch.cat([w["sh_down"][0], w["sh_down"][1]], dim=1)
    ref, ref_s = blocks_exactly(down[None])
    assert torch.equal(q["sh_down"][..., :144].double(), ref[0]) and torch.equal(q["sh_s_down"], ref_s[0])
    ref, ref_s = blocks_exactly(w["sh_up"].reshape(1, 144, 136))
    assert torch.equal(q["sh_up"][..., :136].double(), ref[0]) and torch.equal(q["sh_s_up"], ref_s[0])


FFN = [dict(T=1, H=64, E=4, k=1, I=64, E_local=4), dict(T=7, H=264, E=8, k=2, I=136, E_local=8, n_shared=1, I_shared=72),
       dict(T=64, H=512, E=16, k=4, I=256, E_local=6, n_shared=2, I_shared=136), dict(T=300, H=1000, E=12, k=3, I=520, E_local=12),
       dict(T=1030, H=1024, E=8, k=2, I=776, E_local=5, n_shared=1, I_shared=264), dict(T=2100, H=640, E=32, k=4, I=384, E_local=32),
       dict(T=3, H=2048, E=64, k=6, I=1408, E_local=64, n_shared=2, I_shared=1408)]


def dispatch(moe, d, seed):
    """Offsets of a skewed dispatch of T k pairs, some slots without rows."""
    rng = np.random.default_rng(seed)
    p = rng.random(d.E) ** 2 * (rng.random(d.E) < 0.85) + 1e-6
    rows = rng.multinomial(d.T * d.k, p / p.sum())[:d.E_local]
    rows = np.minimum(rows, d.T)
    return np.concatenate([[0], np.cumsum(rows)]).tolist()


def expert(q, e, p="w_", ps="s_"):
    at = (lambda t: t) if e is None else (lambda t: t[e])
    return [(at(q[p + n]), at(q[ps + n])) for n in ("gate", "up", "down")]


def assert_ffn(y, x, w):
    ref, bound = ffn_and_bound(x, *w)
    off = (y.double() - ref).abs()
    assert (off <= bound).all(), (off / bound).max().item()


@pytest.mark.parametrize("case", range(len(FFN)))
def test_expert_ffn(moe, case):
    d = moe.dims(S=1, **FFN[case])
    _, q = layer_weights(moe, d, case)
    o = dispatch(moe, d, case)
    x_perm, x = randn((d.T * d.k, d.H), case + 50), randn((d.T, d.H), case + 51)
    y = torch.full((d.T * d.k, d.H), 3.0, dtype=torch.bfloat16, device="cuda")
    ysh = torch.full((d.T, d.H), 3.0, dtype=torch.bfloat16, device="cuda") if d.n_shared else None
    ws = moe.workspace(d, moe.ENTRY_EXPERT_FFN_F8).fill_(0xff)
    moe.expert_ffn_f8(d, x_perm, torch.tensor(o, dtype=torch.int32, device="cuda"), moe.make_weights_f8(d, q), x, y, ysh, ws)
    for e in range(d.E_local):
        if o[e] < o[e + 1]:
            assert_ffn(y[o[e]:o[e + 1]], x_perm[o[e]:o[e + 1]], expert(q, e))
    assert (y[o[-1]:] == 3.0).all()
    if d.n_shared:
        assert_ffn(ysh, x, expert(q, None, "sh_", "sh_s_"))


def run_steps(moe, d, logits, src, x, local, w, gating, counts):
    """The layer through its separate entry points, rows gathered."""
    rows, i32, bf = d.T * d.k, dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
    idx, gates = torch.empty((d.T, d.k), **i32), torch.empty((d.T, d.k), device="cuda")
    off, perm, inv = torch.empty(d.E_local + 1, **i32), torch.empty(rows, **i32), torch.empty(rows, **i32)
    xp, yp, out = torch.empty((rows, d.H), **bf), torch.empty((rows, d.H), **bf), torch.empty((d.T, d.H), **bf)
    ysh = torch.empty((d.T, d.H), **bf) if d.n_shared else None
    moe.route(d, logits, idx, gates, gating=gating)
    moe.route_stats(d, src, idx, counts)
    moe.permute(d, idx, local, x, off, perm, inv, xp, moe.workspace(d, moe.ENTRY_PERMUTE))
    moe.expert_ffn_f8(d, xp, off, w, x, yp, ysh, moe.workspace(d, moe.ENTRY_EXPERT_FFN_F8))
    moe.combine(d, yp, inv, gates, ysh, out)
    return out


def placed(d, seed):
    return None if d.E_local == d.E else torch.randperm(d.E, generator=gen(seed), device="cuda")[:d.E_local].to(torch.int32)


def assert_layer(moe, out, d, q, logits, x, local, gating):
    """A layer's output against 64 bits, expert by expert: an expert's output is within
    its bound and the sum adds k + 1 terms in fp32."""
    idx, gates = torch.empty((d.T, d.k), dtype=torch.int32, device="cuda"), torch.empty((d.T, d.k), device="cuda")
    moe.route(d, logits, idx, gates, gating=gating)
    ref, bound = torch.zeros((2, d.T, d.H), dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(ref)
    for slot, e in enumerate(range(d.E) if local is None else local.tolist()):
        t, j = (idx == e).nonzero(as_tuple=True)
        if len(t):
            y, b = ffn_and_bound(x[t], *expert(q, slot))
            g = gates[t, j].double()[:, None]
            ref[t], bound[t], terms[t] = ref[t] + g * y, bound[t] + g * b, terms[t] + g * (y.abs() + b)
    if d.n_shared:
        y, b = ffn_and_bound(x, *expert(q, None, "sh_", "sh_s_"))
        ref, bound, terms = ref + y, bound + b, terms + y.abs() + b
    bound = bound + terms * (d.k + 2) * 2.0 ** -24
    off = (out.double() - ref).abs()
    bound = bound + (ref.abs() + bound) * BF16
    assert (off <= bound).all(), (off / bound).max().item()


@pytest.mark.parametrize("case", range(len(FFN)))
def test_forward_is_its_steps(moe, case):
    """forward_f8 gives the bits of route, permute, expert_ffn_f8 and combine, and
    the layer class those of forward_f8; the counts are those of the steps.  From
    quantised rows too, but that with up to 8 tokens other kernels add in another
    order: those are held against 64 bits."""
    d = moe.dims(S=3, flags=case % 3, **FFN[case])
    _, q = layer_weights(moe, d, case)
    logits, x = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), case + 60)
    src = torch.randint(0, 3, (d.T,), generator=gen(case), device="cuda", dtype=torch.int32)
    local = placed(d, case)
    gating = moe.gating(None, 1.5)
    counts = [torch.zeros((3, d.E), dtype=torch.int64, device="cuda") for _ in range(3)]
    ref = run_steps(moe, d, logits, src, x, local, moe.make_weights_f8(d, q), gating, counts[0])
    layer = moe.MoeLayerF8(d, q, local, gating=gating)
    out = layer.forward(logits, src, x, counts=counts[1])
    assert torch.equal(out, ref) and torch.equal(counts[0], counts[1])
    xq, xs = moe.quantize_rows_f8(x)
    out = layer.forward(logits, src, counts=counts[2], xq=xq, x_scale=xs)
    assert torch.equal(counts[0], counts[2])
    if d.T > 8:
        assert torch.equal(out, ref)
    else:
        assert_layer(moe, out, d, q, logits, x, local, gating)
        assert_layer(moe, ref, d, q, logits, x, local, gating)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = layer.forward(logits, src, x, stream=side, ws=moe.workspace(d, moe.ENTRY_FORWARD_F8).fill_(0xff))
    side.synchronize()
    assert torch.equal(again, ref)


def test_layer_from_bf16_weights_is_close_to_the_bf16_layer(moe):
    """What 8 bits cost: the layer's output against MoeLayer's on the same weights.
    Rounding to 4 significant bits errs by up to 1/16 to 1/32 of a value, evenly:
    1/32 / sqrt(3) * 1.44 = 2.6 % by norm for x, for a weight and for h; of a sum
    of independent products each factor's share stays what it is: gate and up 3.7 %
    each, their product 5.2 % at most twice over (silu's slope), with h and down's own
    6.4 %."""
    d = moe.dims(256, 1024, 8, 2, 512, 1, 8, 1, 256)
    w, _ = layer_weights(moe, d, 3)
    logits, x = torch.randn((d.T, d.E), generator=gen(1), device="cuda"), randn((d.T, d.H), 2)
    a = moe.MoeLayer(d, w).forward(logits, None, x).double()
    b = moe.MoeLayerF8(d, w).forward(logits, None, x).double()
    assert ((a - b).norm() / a.norm()).item() < 0.09


@pytest.mark.parametrize("case", [0, 2, 4, 5])
def test_layer_in_a_graph(moe, case):
    """Captured once, replayed with new inputs among eager calls of the same layer."""
    d = moe.dims(S=1, **FFN[case])
    _, q = layer_weights(moe, d, case)
    layer = moe.MoeLayerF8(d, q, placed(d, 1))
    logits, x = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), case)
    out, ws = torch.empty_like(x), moe.workspace(d, moe.ENTRY_FORWARD_F8)
    layer.forward(logits, None, x, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(logits, None, x, out=out, ws=ws)
    for seed in range(4):
        logits.normal_(generator=gen(seed))
        x.copy_(randn((d.T, d.H), seed + 9))
        eager = layer.forward(logits, None, x)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), seed


def test_nan_rows_stay_their_own(moe):
    """A token with a NaN gives NaN outputs for itself and none for others."""
    d = moe.dims(T=40, S=1, H=264, E=4, k=2, I=136, E_local=4, n_shared=1, I_shared=32)
    _, q = layer_weights(moe, d, 1)
    layer = moe.MoeLayerF8(d, q)
    logits, x = torch.randn((40, 4), generator=gen(1), device="cuda"), randn((40, 264), 3)
    ref = layer.forward(logits, None, x)
    x2 = x.clone()
    x2[7, 5], x2[9, 263] = float("nan"), float("inf")
    x2[11] = 0.0
    out = layer.forward(logits, None, x2)
    assert torch.isnan(out[[7, 9]]).all() and (out[11] == 0).all()
    keep = [t for t in range(40) if t not in (7, 9, 11)]
    assert torch.equal(out[keep], ref[keep])


def test_no_tokens(moe):
    d = moe.dims(T=0, S=1, H=64, E=4, k=2, I=64, E_local=4, n_shared=1, I_shared=32)
    _, q = layer_weights(moe, d, 1)
    e = dict(dtype=torch.bfloat16, device="cuda")
    counts = torch.ones((1, 4), dtype=torch.int64, device="cuda")
    out = moe.MoeLayerF8(d, q).forward(torch.empty((0, 4), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                                       torch.empty((0, 64), **e), counts=counts)
    torch.cuda.synchronize()
    assert out.shape == (0, 64) and (counts == 1).all()


@pytest.mark.parametrize("sizes", [[24, 0, 0], [0, 9, 15], [17, 0, 1], [0, 0, 0], [1, 1, 1]])
def test_few_tokens_in_any_groups(moe, sizes):
    """expert_ffn_f8 of 8 tokens, however their rows lie; rows behind the last
    group stay as they were."""
    d = moe.dims(T=8, S=1, H=264, E=3, k=3, I=200, E_local=3, n_shared=1, I_shared=88)
    _, q = layer_weights(moe, d, 5)
    w = moe.make_weights_f8(d, q)
    o = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    x_perm, x = randn((24, d.H), 1), randn((8, d.H), 2)
    y = torch.full((24, d.H), 3.0, dtype=torch.bfloat16, device="cuda")
    ysh = torch.empty((8, d.H), dtype=torch.bfloat16, device="cuda")
    ws = moe.workspace(d, moe.ENTRY_EXPERT_FFN_F8).fill_(0xff)
    moe.expert_ffn_f8(d, x_perm, torch.tensor(o, dtype=torch.int32, device="cuda"), w, x, y, ysh, ws)
    for e in range(3):
        if o[e] < o[e + 1]:
            assert_ffn(y[o[e]:o[e + 1]], x_perm[o[e]:o[e + 1]], expert(q, e))
    assert (y[o[-1]:] == 3.0).all()
    assert_ffn(ysh, x, expert(q, None, "sh_", "sh_s_"))


# Few tokens: the products quantise the rows themselves, K in four, two and one
# parts, rows longer than the registers hold (down, 9000), rows of the last case too
# long for it at 8 tokens, and a shared expert of its own width.
FEW = [dict(H=512, E=16, k=2, I=256, E_local=16), dict(H=2048, E=32, k=4, I=768, E_local=24),
       dict(H=1000, E=6, k=3, I=1544, E_local=6, n_shared=1, I_shared=344), dict(H=136, E=8, k=8, I=40, E_local=8),
       dict(H=256, E=4, k=2, I=9000, E_local=4, n_shared=2, I_shared=1000), dict(H=4104, E=8, k=4, I=2056, E_local=8),
       dict(H=8704, E=2, k=1, I=264, E_local=2)]


@pytest.mark.parametrize("case", range(len(FEW)))
def test_few_tokens(moe, case):
    """Up to 9 tokens, from bf16 rows and from quantised ones; one row is zero and
    one not finite."""
    big = moe.dims(T=9, S=1, **FEW[case])
    _, q = layer_weights(moe, big, case)
    local = None if big.E_local == big.E else torch.arange(big.E_local, dtype=torch.int32, device="cuda")
    logits, x = torch.randn((9, big.E), generator=gen(case), device="cuda"), randn((9, big.H), case)
    x[1], x[4, 3] = 0.0, float("nan")
    for T in (1, 2, 3, 5, 8, 9):
        d = moe.dims(T=T, S=1, **FEW[case])
        layer = moe.MoeLayerF8(d, q, local)
        xq, xs = moe.quantize_rows_f8(x[:T])
        for rows in (dict(x=x[:T]), dict(xq=xq, x_scale=xs)):
            layer.ws.fill_(0xff)
            out = layer.forward(logits[:T], None, **rows)
            # (a token none of whose experts is hosted here, without shared ones, is zero)
            keep = [t for t in range(T) if t != 4]
            at = moe.dims(T=len(keep), S=1, **FEW[case])
            assert_layer(moe, out[keep], at, q, logits[keep], x[keep], local, None)
            if T > 4:
                assert torch.isnan(out[4]).all() or (out[4] == 0).all()


# --------------------------------------------- far offsets, calls at once ----


def random_f8(shape, seed):
    """Random e4m3 of magnitudes up to 1.875."""
    b = torch.randint(0, 256, shape, generator=gen(seed), device="cuda", dtype=torch.uint8)
    return (b & 0xbf).view(F8)


@pytest.mark.parametrize("K", [32, 400])
def test_linear_past_32_bit_offsets(moe, K):
    """More than 2^31 results: 4 GB of them, rows of the first, a middle and the last tile."""
    M, N = 66003, 33001
    xq, wq = random_f8((M, pad16(K)), K), random_f8((N, pad16(K)), K + 1)
    xs, ws = torch.rand((M, blocks(K)), generator=gen(1), device="cuda"), torch.rand((blocks(N), blocks(K)), generator=gen(2), device="cuda")
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    moe.linear_f8(K, xq, xs, wq, ws, y)
    for r in (slice(0, 3), slice(32767, 32770), slice(M - 3, M)):
        assert_product(y[r], xq[r], xs[r], wq, ws, K)


@pytest.mark.parametrize("rows", [1, 90])
def test_grouped_past_32_bit_offsets(moe, rows):
    """2.6 GB of weights; the first, a middle and the last group."""
    G, N, K = 320, 1000, 8200
    M = G * rows
    xq, wq = random_f8((M, pad16(K)), rows), random_f8((G, N, pad16(K)), rows + 1)
    raw(xq)[:, K:], raw(wq)[:, :, K:] = 0, 0  # rows go on with zeros
    xs = torch.rand((M, blocks(K)), generator=gen(1), device="cuda")
    ws = torch.rand((G, blocks(N), blocks(K)), generator=gen(2), device="cuda")
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    offsets = torch.arange(0, M + 1, rows, dtype=torch.int32, device="cuda")
    moe.grouped_linear_f8(K, xq, xs, offsets, wq, ws, y)
    for e in (0, 261, 262, G - 1):
        r = slice(e * rows, e * rows + rows)
        assert_product(y[r], xq[r], xs[r], wq[e], ws[e], K)


def test_quantize_more_rows_than_workgroups(moe):
    """Workgroups that take several lots of rows in turn."""
    rows = 2 ** 26 + 3
    x = torch.empty((rows, 8), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(5))
    q, scale = moe.quantize_rows_f8(x)
    for r in (slice(0, 70), slice(rows - 70, rows), slice(2 ** 26 - 70, 2 ** 26)):
        ref, ref_s = rows_exactly(x[r])
        assert torch.equal(q[r, :8].double(), ref) and torch.equal(scale[r], ref_s) and (raw(q)[r, 8:] == 0).all()


def test_quantize_past_32_bit_offsets(moe):
    rows, cols = 140001, 16400
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(5))
    q, scale = moe.quantize_rows_f8(x)
    for r in (slice(0, 2), slice(65484, 65487), slice(130943, 130946), slice(rows - 2, rows)):
        ref, ref_s = rows_exactly(x[r])
        assert torch.equal(q[r].double(), ref) and torch.equal(scale[r], ref_s)
    q, scale = moe.quantize_blocks_f8(x)
    ref, ref_s = blocks_exactly(x[None, rows - rows % 128:])
    assert torch.equal(q[rows - rows % 128:].double(), ref[0]) and torch.equal(scale[-1], ref_s[0, 0])


@pytest.mark.parametrize("gather", [False, True])
def test_expected_rows_move_no_result(moe, gather):
    """Room for four times the rows: the expected number chooses the kernel (told
    nothing, that of all the room); rows behind the last group stay as they were."""
    sizes, N, K = ragged(24, 75, 3), 1100, 1600
    M, xq, xs, wq, ws, offsets, x_rows = grouped_case(sizes, N, K, 7, spare=4 * sum(sizes), gather=500 if gather else None)
    o, kernels = offsets.tolist(), set()
    for rows in (None, sum(sizes), 1, M, 24 * 75, -3):
        d, out = moe.MoeLinearDims(M=M, N=N, K=K, G=24, R=rows or 0), (C.c_int64 * 4)()
        assert moe._lib.moe_test_linear_f8_plan(C.byref(d), 1, out) == 0
        kernels.add(out[0])
        y = torch.full((M, N), 3.0, dtype=torch.bfloat16, device="cuda")
        moe.grouped_linear_f8(K, xq, xs, offsets, wq, ws, y, x_rows=x_rows, rows=rows)
        assert (y[o[-1]:] == 3.0).all(), rows
        for g in range(24):
            if o[g] < o[g + 1]:
                assert_product(y[o[g]:o[g + 1]], xq, xs, wq[g], ws[g], K, slice(o[g], o[g + 1]) if x_rows is None else x_rows[o[g]:o[g + 1]].long())
    assert kernels == {ITEMS, TILES}


@pytest.mark.parametrize("case", [1, 5])
def test_taps_of_the_layer(moe, case):
    """The extra outputs are those of the separate steps, the output that of the
    layer without them; events of every stage are recorded in order."""
    d = moe.dims(S=3, **FFN[case])
    _, q = layer_weights(moe, d, case)
    logits, x = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), case + 60)
    src = torch.randint(0, 3, (d.T,), generator=gen(case), device="cuda", dtype=torch.int32)
    local = torch.randperm(d.E, generator=gen(case), device="cuda")[:d.E_local].to(torch.int32)
    rows, i32 = d.T * d.k, dict(dtype=torch.int32, device="cuda")

    def outputs():
        return dict(topk_idx=torch.full((d.T, d.k), -7, **i32), topk_w=torch.full((d.T, d.k), -7.0, device="cuda"),
                    expert_load=torch.full((d.E,), -7, **i32), offsets=torch.full((d.E_local + 1,), -7, **i32),
                    perm_token=torch.full((rows,), -7, **i32), inv_pos=torch.full((rows,), -7, **i32))
    ref, got = outputs(), outputs()
    counts = [torch.zeros((3, d.E), dtype=torch.int64, device="cuda") for _ in range(2)]
    moe.route(d, logits, ref["topk_idx"], ref["topk_w"])
    moe.route_stats(d, src, ref["topk_idx"], counts[0], ref["expert_load"])
    moe.permute(d, ref["topk_idx"], local, None, ref["offsets"], ref["perm_token"], ref["inv_pos"], None,
                moe.workspace(d, moe.ENTRY_PERMUTE))
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2 * len(moe.STAGES))]
    for e in events:
        e.record()   # (torch makes the handle with the first record)
    layer = moe.MoeLayerF8(d, q, local)
    plain = layer.forward(logits, src, x)
    h, norm = randn((d.T, d.H), 3), moe.norm(d.H)
    ends = [torch.empty_like(h) for _ in range(2)]
    layer.forward(logits, src, x, norm=norm, rows=moe.norm_io(h, ends[0]))
    out = torch.empty_like(plain)
    layer.forward(logits, src, x, counts=counts[1], out=out, norm=norm, rows=moe.norm_io(h, ends[1]),
                  taps=moe.make_taps(**got, events=[e.cuda_event for e in events]))
    torch.cuda.synchronize()
    assert torch.equal(out, plain) and torch.equal(*ends) and torch.equal(*counts)
    used = ref["offsets"][-1].item()
    for name in got:
        n = used if name == "perm_token" else None
        assert torch.equal(got[name].flatten()[:n], ref[name].flatten()[:n]), name
    assert all(a.elapsed_time(b) >= 0 for a, b in zip(events, events[1:]))


@pytest.mark.parametrize("T", [3, 200])
def test_two_streams_at_once(moe, T):
    """One layer on two streams, each with a workspace of its own."""
    d = moe.dims(T=T, S=1, H=1024, E=16, k=2, I=520, E_local=16, n_shared=1, I_shared=264)
    _, q = layer_weights(moe, d, 2)
    layer = moe.MoeLayerF8(d, q)
    data = [(torch.randn((T, 16), generator=gen(s), device="cuda"), randn((T, 1024), s)) for s in range(2)]
    ref = [layer.forward(lg, None, x) for lg, x in data]
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [moe.workspace(d, moe.ENTRY_FORWARD_F8) for _ in range(2)]
    out = [[torch.empty_like(ref[0]) for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for s in range(2):
            layer.forward(data[s][0], None, data[s][1], out=out[s][i], stream=streams[s], ws=ws[s])
    torch.cuda.synchronize()
    for s in range(2):
        assert all(torch.equal(o, ref[s]) for o in out[s])


def test_outputs_on_a_raw_stream_handle(moe):
    """Allocated outputs belong to the stream that writes them, given as a handle too."""
    d = moe.dims(T=6000, S=1, H=1048, E=4, k=2, I=64, E_local=4)
    _, q = layer_weights(moe, d, 1)
    layer, side = moe.MoeLayerF8(d, q), torch.cuda.Stream()
    logits, x, wide = torch.randn((6000, 4), generator=gen(1), device="cuda"), randn((6000, 1048), 3), randn((6000, 2100), 4)
    eager, (eq, es) = layer.forward(logits, None, x), moe.quantize_rows_f8(wide)
    for handle in (side.cuda_stream, C.c_void_p(side.cuda_stream)):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        out, (xq, xs) = layer.forward(logits, None, x, stream=handle), moe.quantize_rows_f8(wide, stream=handle)
        side.synchronize()
        assert torch.equal(out, eager) and torch.equal(raw(xq), raw(eq)) and torch.equal(xs, es)
        made = {out.data_ptr(), xq.data_ptr()}
        torch.cuda.synchronize()   # (the comparisons read them on the current stream)
        del out, xq, xs
        other = [torch.empty(12 << 20, dtype=torch.uint8, device="cuda") for _ in range(4)]
        with torch.cuda.stream(side):
            own = [torch.empty(12 << 20, dtype=torch.uint8, device="cuda") for _ in range(4)]
        assert made <= {t.data_ptr() for t in own} and not made & {t.data_ptr() for t in other}


# ------------------------------------------ shapes that reach each kernel ----


ITEMS, TILES, FEWS, HALF = 0, 1, 2, "half"


def linear_plan(moe, M, N, K, G=0):
    """(kernel, parts of K, rows of a tile or chunk), and HALF where a wave
    takes 16 weight rows."""
    d, out = moe.MoeLinearDims(M=M, N=N, K=K, G=G), (C.c_int64 * 4)()
    assert moe._lib.moe_test_linear_f8_plan(C.byref(d), int(G > 0), out) == 0
    return tuple(out[:3]) + ((HALF,) if out[3] else ())


# Items: few rows with K in 2 and 4 parts, chunks of 64, 32 and 8, a wave with 32
# and 16 weight rows; undivided, with 256 weight rows per item.  Tiles: last rounds in
# parts and whole, K a byte past the items', more than 64 stages.
KERNELS = [(7, 9001, 130, (ITEMS, 2, 8)), (8, 517, 1003, (ITEMS, 4, 8, HALF)), (50, 1003, 517, (ITEMS, 4, 32, HALF)),
           (7, 5001, 1003, (ITEMS, 4, 8)), (50, 4001, 517, (ITEMS, 4, 32)), (30, 1999, 1700, (ITEMS, 4, 32, HALF)),
           (260, 300, 3001, (ITEMS, 4, 32, HALF)), (50, 5003, 517, (ITEMS, 4, 64)), (60, 12003, 4100, (ITEMS, 2, 64)),
           (777, 1003, 517, (ITEMS, 2, 64)), (4200, 2051, 380, (ITEMS, 1, 128)), (100, 33000, 8200, (TILES, 1, 192)),
           (50, 17000, 517, (ITEMS, 1, 128)), (150, 6001, 1300, (ITEMS, 2, 64)), (5, 8200, 34000, (ITEMS, 2, 8)), (3, 300, 130000, (ITEMS, 4, 8, HALF)),
           (2500, 2100, 1700, (TILES, 1, 192)), (5003, 3801, 1501, (TILES, 1, 192)), (5003, 2803, 1501, (TILES, 1, 192)),
           (16000, 1027, 385, (TILES, 1, 192)), (2600, 2049, 8200, (TILES, 1, 192)), (1900, 2304, 12288, (TILES, 1, 192)),
           (1350, 1500, 16500, (TILES, 1, 192)), (193, 7300, 641, (ITEMS, 2, 64)),
           (300, 14600, 641, (TILES, 1, 192)), (400, 4100, 700, (ITEMS, 2, 64)), (16000, 60, 500, (ITEMS, 2, 64))]


@pytest.mark.parametrize("M,N,K,plan", KERNELS)
def test_linear_kernels(moe, M, N, K, plan):
    assert linear_plan(moe, M, N, K) == plan
    xq, xs, wq, ws = operands(M, N, K, M + N + K)
    y = torch.full((M + 1, N), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.linear_f8(K, xq, xs, wq, ws, y[:M])
    for a in range(0, M, 1000):
        assert_product(y[a:min(M, a + 1000)], xq[a:a + 1000], xs[a:a + 1000], wq, ws, K)
    assert (y[M] == 3.0).all()


# Groups: tiles of up to 64, 256 and 1024 groups with their last tiles in each of
# their forms, empty groups and one that has most rows; items.
GROUP_KERNELS = [(ragged(8, 350, 1), 2000, 1600, (TILES, 1, 192)),
                 ([0, 64, 65, 96, 97, 192, 193, 2800, 0, 33, 32], 1999, 1603, (TILES, 1, 192)),
                 (ragged(100, 120, 2, 1500), 513, 2100, (TILES, 1, 192)), (ragged(300, 120, 3), 260, 2100, (TILES, 1, 192)),
                 (ragged(1000, 110, 4), 70, 2052, (TILES, 1, 192)), (ragged(140, 36, 7), 1030, 900, (TILES, 1, 192)),
                 (ragged(30, 16, 5, 600), 1003, 900, (ITEMS, 1, 128)), ([5, 0, 70, 3], 3000, 700, (ITEMS, 2, 64)),
                 ([2, 0, 1], 1000, 700, (ITEMS, 4, 8, HALF)), ([2, 30, 0, 9], 600, 900, (ITEMS, 4, 32, HALF)),
                 ([2, 70, 0, 9, 33, 32, 8], 100, 900, (ITEMS, 4, 32, HALF)), ([3, 0, 4, 1], 2500, 500, (ITEMS, 2, 8)),
                 (ragged(12, 60, 5), 1500, 1100, (ITEMS, 2, 64)), (ragged(24, 30, 6), 1003, 1100, (ITEMS, 1, 128)), (ragged(9, 200, 8), 700, 1500, (ITEMS, 2, 64)),
                 (ragged(40, 60, 9), 3000, 2300, (ITEMS, 1, 128))]


@pytest.mark.parametrize("case", range(len(GROUP_KERNELS)))
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_kernels(moe, case, gather):
    sizes, N, K, plan = GROUP_KERNELS[case]
    assert linear_plan(moe, sum(sizes), N, K, len(sizes)) == plan
    check_grouped(moe, sizes, N, K, case, spare=0, gather=max(1, sum(sizes) // 3) if gather else None)


def ffn_plan(moe, d, quantised=False):
    out = (C.c_int64 * 8)()
    assert moe._lib.moe_test_ffn_f8_plan(C.byref(d), int(quantised), out) == 0
    return tuple(out[:3]), tuple(out[4:7])


FFN_KERNELS = [(dict(T=1500, H=1600, E=4, k=2, I=1032, E_local=4, n_shared=1, I_shared=520), (TILES, 1, 192), (TILES, 1, 192)),
               (dict(T=3300, H=2104, E=80, k=3, I=136, E_local=70), (TILES, 1, 192), (ITEMS, 1, 128)),
               (dict(T=7200, H=2104, E=300, k=4, I=136, E_local=300), (TILES, 1, 192), (ITEMS, 1, 128)),
               (dict(T=3000, H=256, E=4, k=2, I=1536, E_local=4), (ITEMS, 1, 128), (ITEMS, 2, 64)),
               (dict(T=2000, H=2048, E=4, k=2, I=1544, E_local=4, n_shared=1, I_shared=1600), (TILES, 1, 192), (TILES, 1, 192)),
               (dict(T=5000, H=1160, E=16, k=3, I=904, E_local=16, n_shared=2, I_shared=456), (TILES, 1, 192), (TILES, 1, 192)),
               (dict(T=8, H=1024, E=8, k=2, I=520, E_local=8, n_shared=1, I_shared=264), (FEWS, 2, 8), (FEWS, 2, 8)),
               # few routed rows beside a wide shared network
               (dict(T=2000, H=1032, E=64, k=2, I=520, E_local=4, n_shared=1, I_shared=2056), (TILES, 1, 192), (TILES, 1, 192)),
               # gate and up in every cut of the items: K in two parts, a workgroup per CU and two, in four, whole
               (dict(T=60, H=1032, E=4, k=2, I=1160, E_local=4), (ITEMS, 2, 64), (ITEMS, 4, 64)),
               (dict(T=300, H=1032, E=4, k=2, I=520, E_local=4), (ITEMS, 2, 64), (ITEMS, 2, 64)),
               (dict(T=150, H=520, E=2, k=1, I=72, E_local=2, n_shared=1, I_shared=1288), (ITEMS, 2, 64), (ITEMS, 4, 64)),
               (dict(T=400, H=1032, E=4, k=2, I=904, E_local=4), (ITEMS, 2, 64), (ITEMS, 2, 64)),
               (dict(T=100, H=1032, E=4, k=1, I=264, E_local=4), (ITEMS, 4, 32), (ITEMS, 4, 64)),
               (dict(T=100, H=1032, E=4, k=1, I=776, E_local=4), (ITEMS, 4, 64), (ITEMS, 4, 64)),
               (dict(T=100, H=1032, E=16, k=2, I=1032, E_local=16), (ITEMS, 1, 128), (ITEMS, 1, 128))]


@pytest.mark.parametrize("case", range(len(FFN_KERNELS)))
def test_ffn_kernels(moe, case):
    """The layers that tiles and wide items are for, and their bits from one
    entry point to the other."""
    conf, up, down = FFN_KERNELS[case]
    d = moe.dims(S=1, **conf)
    assert ffn_plan(moe, d) == (up, down)
    _, q = layer_weights(moe, d, case)
    w = moe.make_weights_f8(d, q)
    local = None if d.E_local == d.E else torch.arange(d.E_local, dtype=torch.int32, device="cuda")
    logits, x = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), case)
    out = moe.MoeLayerF8(d, q, local).forward(logits, None, x)
    src, counts = torch.zeros(d.T, dtype=torch.int32, device="cuda"), torch.zeros((1, d.E), dtype=torch.int64, device="cuda")
    assert torch.equal(out, run_steps(moe, d, logits, src, x, local, w, None, counts))
    # and the experts' rows against 64 bits
    o = dispatch(moe, d, case)
    x_perm = randn((d.T * d.k, d.H), case + 50)
    y = torch.full((d.T * d.k, d.H), 3.0, dtype=torch.bfloat16, device="cuda")
    ysh = torch.empty((d.T, d.H), dtype=torch.bfloat16, device="cuda") if d.n_shared else None
    moe.expert_ffn_f8(d, x_perm, torch.tensor(o, dtype=torch.int32, device="cuda"), w, x, y, ysh,
                      moe.workspace(d, moe.ENTRY_EXPERT_FFN_F8).fill_(0xff))
    for e in range(0, d.E_local, max(1, d.E_local // 8)):
        if o[e] < o[e + 1]:
            assert_ffn(y[o[e]:o[e + 1]], x_perm[o[e]:o[e + 1]], expert(q, e))
    assert (y[o[-1]:] == 3.0).all()
    if d.n_shared:
        assert_ffn(ysh, x, expert(q, None, "sh_", "sh_s_"))


# Rows of up to 8 tokens that come quantised: gate and up in chunks of 8, K in four,
# two and one parts, and the kernel that down has.
QUANTISED = [(dict(T=8, H=1032, E=4, k=2, I=264, E_local=4), (ITEMS, 4, 8), (FEWS, 4, 8)),
             (dict(T=8, H=1032, E=4, k=2, I=1160, E_local=4), (ITEMS, 2, 8), (FEWS, 4, 8)),
             (dict(T=5, H=1000, E=6, k=3, I=1544, E_local=6, n_shared=1, I_shared=344), (ITEMS, 1, 128), (FEWS, 4, 5)),
             (dict(T=5, H=256, E=4, k=2, I=9000, E_local=4), (ITEMS, 1, 128), (ITEMS, 4, 8))]


@pytest.mark.parametrize("case", range(len(QUANTISED)))
def test_quantised_rows_of_few_tokens(moe, case):
    conf, up, down = QUANTISED[case]
    d = moe.dims(S=1, **conf)
    assert ffn_plan(moe, d, quantised=True) == (up, down)
    _, q = layer_weights(moe, d, case)
    logits, x = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), case)
    xq, xs = moe.quantize_rows_f8(x)
    layer = moe.MoeLayerF8(d, q)
    layer.ws.fill_(0xff)
    assert_layer(moe, layer.forward(logits, None, xq=xq, x_scale=xs), d, q, logits, x, None, None)


@pytest.mark.parametrize("case", range(len(FEW)))
def test_few_tokens_not_finite(moe, case):
    """A token with a NaN or an infinity is NaN wherever an expert of its picks is hosted
    or there is a shared one, and zero elsewhere; no other token changes."""
    big = moe.dims(T=9, S=1, **FEW[case])
    _, q = layer_weights(moe, big, case)
    local = None if big.E_local == big.E else torch.arange(big.E_local, dtype=torch.int32, device="cuda")
    x = randn((9, big.H), case)
    bad = x.clone()
    bad[1, big.H - 1], bad[4, 3] = float("inf"), float("nan")
    for seed in range(3):
        logits = torch.randn((9, big.E), generator=gen(seed), device="cuda")
        if seed == 2:
            logits[1, big.E - big.k:] += 40.0   # (token 1 picks the last experts)
        for T in (2, 5, 8, 9):
            d = moe.dims(T=T, S=1, **FEW[case])
            idx, gates = torch.empty((T, d.k), dtype=torch.int32, device="cuda"), torch.empty((T, d.k), device="cuda")
            moe.route(d, logits[:T], idx, gates)
            hosted = (idx < d.E_local).any(dim=1) | (d.n_shared > 0)
            layer = moe.MoeLayerF8(d, q, local)
            for quantised in (False, True):
                def run(rows):
                    layer.ws.fill_(0xff)
                    if not quantised:
                        return layer.forward(logits[:T], None, rows[:T])
                    xq, xs = moe.quantize_rows_f8(rows[:T])
                    return layer.forward(logits[:T], None, xq=xq, x_scale=xs)
                out, ref = run(bad), run(x)
                for t in range(T):
                    if t not in (1, 4):
                        assert torch.equal(out[t], ref[t]), (T, quantised, t)
                    elif hosted[t]:
                        assert torch.isnan(out[t]).all(), (T, quantised, t)
                    else:
                        assert (out[t] == 0).all(), (T, quantised, t)
    assert hosted[1] == (big.E_local == big.E)   # (both were seen where experts are missing)
