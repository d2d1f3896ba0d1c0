"""The norms around the layer on the GPU, by themselves and as the layer's end,
against their definitions in 64 bits (bounds: f8_util.py)."""
import pytest
import torch

from tests.f8_util import BF16, F8, FP32, blocks, by_column, e4m3_step, gen, norm_and_bounds, pad16, randn, rows_exactly

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    from paper_2606_15177_amd import moe
    return moe


def within(got, ref, bound):
    off = (got.double() - ref).abs()
    assert (off <= bound).all(), (off - bound).max().item()


def assert_rows_of(q, scale, x, ex):
    """q and scale stand for rows within ex of x: the scale is that of their largest,
    a value is half an e4m3 step off at most."""
    T, H = x.shape
    pad = lambda v: torch.nn.functional.pad(v, (0, -H % 128)).view(T, -1, 128)  # noqa: E731
    a, ea = pad(x.abs()).amax(dim=2), pad(ex).amax(dim=2)
    within(scale, a / 448.0, (ea + a * FP32) / 448.0 + 2.0 ** -149)
    s = by_column(scale, H)
    v = q[:, :H].double()
    # 448 x / a: two roundings in fp32 and one to e4m3, of x and a as they came out
    off = (v * s - x).abs()
    slack = ex + (x.abs() + ex) * 4 * FP32
    assert (off <= (0.5 * e4m3_step(v) * (1 + 2.0 ** -9) + 2.0 ** -30) * s + slack * (1 + 2.0 ** -4) + by_column(ea, H)).all()
    assert (q.view(torch.uint8)[:, H:] == 0).all()


GATES = {"none": None, "column": (0, 1), "row": (1, 0), "both": (1, 1)}


def check(moe, T, H, seed, post=True, gate="none", pre=True, quant=True, rho=1.0, add=0.0, with_y=True, pad=0, eps=1e-6, unit=False):
    def vec(shape, k):
        return (1.0 - add + 0.3 * torch.randn(shape, generator=gen(seed + k), device="cuda")).to(torch.bfloat16)

    def rows(k, std):
        return randn((T, H + pad), seed + k, std)[:, pad // 2:pad // 2 + H]
    y, h = rows(0, 1.0) if with_y else None, rows(1, 3.0)
    pw, w = vec((H,), 2) if post else None, vec((H,), 3) if pre and not unit else None
    g = None if GATES[gate] is None else vec(tuple(n if f else 1 for n, f in zip((T, H), GATES[gate])), 4) + add
    out, x = (torch.full((T + 2, H + pad + 3), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.full((T, pad16(H) + 32), 77, dtype=torch.uint8, device="cuda")
    scale = torch.full((T + 1, blocks(H)), 5.0, device="cuda")
    io = moe.norm_io(h, out[1:T + 1, 1:H + 1], x=x[1:T + 1, 2:H + 2] if pre else None,
                     q=q[:, 16:16 + pad16(H)].view(F8) if pre and quant else None, scale=scale[:T] if pre and quant else None, gate=g)
    keep = h.clone()
    moe.norm_rows(moe.norm(H, w, pw, rho, eps, add), io, y=y)
    (rh, bh), (rx, bx, ex) = norm_and_bounds(y, h, pw, g, w, rho, eps, add)
    within(out[1:T + 1, 1:H + 1], rh, bh)
    assert torch.equal(h, keep)
    edge = out.clone()
    edge[1:T + 1, 1:H + 1] = 7.0
    assert (edge == 7.0).all()
    if pre:
        within(x[1:T + 1, 2:H + 2], rx, bx)
        edge = x.clone()
        edge[1:T + 1, 2:H + 2] = 7.0
        assert (edge == 7.0).all()
        if quant:
            assert_rows_of(q[:, 16:16 + pad16(H)].view(F8), scale[:T], rx, ex)
            assert (scale[T] == 5.0).all() and (q[:, :16] == 77).all() and (q[:, 16 + pad16(H):] == 77).all()


@pytest.mark.parametrize("T,H", [(1, 1), (1, 7), (3, 8), (2, 64), (5, 129), (4, 511), (4, 512), (3, 513), (2, 1000), (70, 2048), (3, 2049),
                                 (1, 7168), (9, 4099), (3, 8192), (2, 8193), (1, 16384), (2, 20001), (2, 32768), (1500, 264),
                                 (700, 4096), (700, 3001), (600, 7168), (530, 8190), (600, 16000)])
def test_norm_sizes(moe, T, H):
    check(moe, T, H, T + H)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", list(GATES))
@pytest.mark.parametrize("pre,quant", [(False, False), (True, False), (True, True)])
def test_norm_forms(moe, post, gate, pre, quant):
    check(moe, 5, 1003, 3, post=post, gate=gate, pre=pre, quant=quant, rho=0.875)
    check(moe, 40, 136, 4, post=post, gate=gate, pre=pre, quant=quant, rho=-1.5, add=1.0, pad=5)


@pytest.mark.parametrize("H", [40, 1000, 3000, 9000])
def test_first_norm_and_unit_weights(moe, H):
    """Without y: the stream itself; without weights: ones."""
    check(moe, 6, H, 1, with_y=False, post=True, gate="both")   # (neither is looked at)
    check(moe, 6, H, 2, unit=True, pad=8)
    check(moe, 6, H, 3, post=False, unit=True, with_y=False, eps=0.5)


def quantised_of(moe, h, w):
    """(x, q, scale) of the norm of h with weights w, eps 1 and values whose mean of
    squares is below 2^-25: the root is 1, so that x is h w in fp32, which holds the
    product of two bf16 values exactly."""
    T, H = h.shape
    assert h.double().square().mean(dim=1).max() < 2.0 ** -25
    x, q = torch.empty_like(h), torch.zeros((T, pad16(H)), dtype=torch.uint8, device="cuda").view(F8)
    s = torch.empty((T, blocks(H)), device="cuda")
    moe.norm_rows(moe.norm(H, w, eps=1.0), moe.norm_io(h, x=x, q=q, scale=s))
    return x, q, s


def assert_quotients(moe, h, w):
    x, q, s = quantised_of(moe, h, w)
    exact = h.double() if w is None else h.double() * w.double()
    assert torch.equal(x, exact.float().to(torch.bfloat16))
    # x and its largest a have 16 significant bits at most and a tie of e4m3 has 5, so 448 x / a is a tie or 2^-22 of it
    # away: rounded to fp32 (2^-24) it lies on the side of every tie that it is on in exact arithmetic
    rq, rs = rows_exactly(exact)
    assert torch.equal(s, rs)
    off = q[:, :h.shape[1]].double() != rq
    assert not off.any(), off.sum().item()


@pytest.mark.parametrize("H", [128, 1000, 4100, 16400])
def test_norm_quantises_the_rounded_quotient(moe, H):
    """q is 448 x / a rounded to fp32 once and then to e4m3: products of 16 bits."""
    for seed in range(3):
        for small, large in ((2.0 ** -20, 1.0), (2.0 ** -60, 1.0), (2.0 ** -60, 2.0 ** -40), (2.0 ** -15, 2.0 ** 125)):
            assert_quotients(moe, randn((40, H), seed, small), randn((H,), seed + 9, large))
    assert_quotients(moe, randn((600, H), 5, 2.0 ** -20), None)


def test_norm_quantises_ties(moe):
    """Every tie between e4m3 values, against maxima of 448 j for odd j: x = m j has
    448 x / a = m exactly, which goes to the even neighbour.  (m j times 448 / a rounded
    to fp32 is m for most j only.)"""
    ties = [(8 + m + 0.5) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)]
    ties = [v for v in ties if v < 448.0] + [(m + 0.5) * 2.0 ** -9 for m in range(8)]
    assert len(ties) == 126
    row = torch.tensor(ties + [448.0, -448.0], dtype=torch.float64, device="cuda") * 2.0 ** -30
    h = torch.stack([row, -row]).to(torch.bfloat16)
    assert torch.equal(h[0].double(), row)
    j = torch.arange(1, 256, 2, device="cuda")
    for wide in (1, 9):   # (a wave per row, 256 threads)
        for k in j.tolist():
            w = torch.full((128 * wide,), float(k), dtype=torch.bfloat16, device="cuda")
            assert_quotients(moe, h.repeat(1, wide), w)


@pytest.mark.parametrize("T,H", [(1, 264), (300, 1000), (3, 9001)])
def test_norm_in_place(moe, T, H):
    """h_out over h and x over y: the values of separate outputs."""
    y, h = randn((T, H), 1), randn((T, H), 2)
    w, pw = randn((H,), 3), randn((H,), 4)
    n = moe.norm(H, w, pw, 0.5)
    out, x = torch.empty_like(h), torch.empty_like(h)
    moe.norm_rows(n, moe.norm_io(h, out, x=x), y=y)
    moe.norm_rows(n, moe.norm_io(h, h, x=y), y=y)
    assert torch.equal(h, out) and torch.equal(y, x)


def test_norm_rows_that_are_not_finite(moe):
    """A NaN or an infinity takes its own row (its residual by columns), no other;
    a row of zeros stays zero."""
    T, H = 6, 300
    y, h = randn((T, H), 1), randn((T, H), 2)
    n = moe.norm(H, randn((H,), 3), randn((H,), 4))

    def run(y, h):
        out, x, q, s = torch.empty_like(h), torch.empty_like(h), torch.zeros((T, 304), dtype=torch.uint8, device="cuda").view(F8), \
            torch.empty((T, 3), device="cuda")
        moe.norm_rows(n, moe.norm_io(h, out, x=x, q=q, scale=s), y=y)
        return out, x, q.float(), s
    ref = run(y, h)
    y2, h2 = y.clone(), h.clone()
    y2[1, 5], y2[2, 299], h2[3, 7], h2[4, 0] = float("nan"), float("inf"), float("nan"), float("-inf")
    y2[5], h2[5] = 0.0, 0.0
    out, x, q, s = run(y2, h2)
    assert torch.isnan(out[1]).all() and torch.isnan(x[1:4]).all()
    assert torch.isnan(out[2, 299]) and torch.isnan(out[3, 7]) and not torch.isnan(out[3, 8:]).any()
    assert torch.isnan(x[4, 0]) and (x[4, 1:] == 0).all()          # infinity over infinity, and numbers over it
    assert torch.isnan(s[1:4]).all() and (q[1:4] == 0).all()
    for a, b in zip((out, x, q, s), ref):
        assert torch.equal(a[0], b[0]) and (a[5] == 0).all()


def test_norm_no_rows(moe):
    e = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    moe.norm_rows(moe.norm(40), moe.norm_io(e, e, x=torch.empty_like(e)), y=e)


def test_layer_end_without_rows(moe):
    d = moe.dims(T=0, S=1, H=64, E=4, k=2, I=64, E_local=4)
    layer = layer_of(moe, d, 1)
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty((0, 64), dtype=F8, device="cuda"), torch.empty((0, 1), device="cuda")
    io = moe.norm_io(e, e, x=torch.empty_like(e), q=q, scale=s)
    assert layer.forward(torch.empty((0, 4), device="cuda"), None, e, norm=moe.norm(64), rows=io) is None
    assert layer.forward(torch.empty((0, 4), device="cuda"), None, xq=q, x_scale=s, norm=moe.norm(64), rows=io) is None
    torch.cuda.synchronize()


@pytest.mark.parametrize("T,H", [(4 * 2 ** 20 + 5, 8), (2 ** 20 + 3, 1032)])
def test_norm_more_rows_than_workgroups(moe, T, H):
    """Workgroups that take several rows in turn."""
    y, h = (torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(s)) for s in (1, 2))
    w, pw = randn((H,), 3), randn((H,), 4)
    out, x = torch.empty_like(h), torch.empty_like(h)
    moe.norm_rows(moe.norm(H, w, pw, 0.5), moe.norm_io(h, out, x=x), y=y)
    for r in (slice(0, 70), slice(T - 70, T), slice(T // 2, T // 2 + 70)):
        (rh, bh), (rx, bx, _) = norm_and_bounds(y[r], h[r], pw, None, w, 0.5, 1e-6, 0.0)
        within(out[r], rh, bh)
        within(x[r], rx, bx)


def test_norm_of_the_most_rows(moe):
    """2^31 - 1 rows, four of them a workgroup at a time; every row is looked at."""
    T = 2 ** 31 - 1
    few = randn((65537, 1), 1, 2.0)   # (no power of two repeats with it)
    h = few.repeat(T // len(few) + 1, 1)[:T]
    x, w = torch.empty_like(h), randn((1,), 2)
    moe.norm_rows(moe.norm(1, w, eps=0.5), moe.norm_io(h, x=x))
    _, (rx, bx, _) = norm_and_bounds(None, few, None, None, w, 1.0, 0.5, 0.0)
    lot = 256 * len(few)
    rx, bx = rx.repeat(256, 1), bx.repeat(256, 1)
    for a in range(0, T, lot):
        n = min(lot, T - a)
        within(x[a:a + n], rx[:n], bx[:n])


def test_norm_past_32_bit_offsets(moe):
    T, H = 140001, 16400
    h = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(5))
    x, q, s = torch.empty_like(h), torch.empty((T, H), dtype=F8, device="cuda"), torch.empty((T, blocks(H)), device="cuda")
    moe.norm_rows(moe.norm(H), moe.norm_io(h, x=x, q=q, scale=s))
    for r in (slice(0, 2), slice(65484, 65487), slice(130943, 130946), slice(T - 2, T)):
        _, (rx, bx, ex) = norm_and_bounds(None, h[r], None, None, None, 1.0, 1e-6, 0.0)
        within(x[r], rx, bx)
        assert_rows_of(q[r], s[r], rx, ex)


def test_norm_in_a_graph_and_on_streams(moe):
    T, H = 33, 2056
    y, h, w = randn((T, H), 1), randn((T, H), 2), randn((H,), 3)
    n, out, x = moe.norm(H, w, w), torch.empty_like(h), torch.empty_like(h)
    io = moe.norm_io(h, out, x=x)
    moe.norm_rows(n, io, y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.norm_rows(n, io, y=y)
    for seed in range(4):
        y.copy_(randn((T, H), seed + 9))
        eo, ex = torch.empty_like(h), torch.empty_like(h)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        moe.norm_rows(n, moe.norm_io(h, eo, x=ex), y=y, stream=side)
        torch.cuda.synchronize()
        x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eo) and torch.equal(x, ex), seed


# ---------------------------------------------------------- the layer's end ----


ENDS = [dict(T=1, H=264, E=4, k=2, I=136, E_local=4), dict(T=9, H=1000, E=12, k=3, I=264, E_local=5, n_shared=1, I_shared=72),
        dict(T=300, H=2056, E=8, k=8, I=136, E_local=8, n_shared=2, I_shared=136), dict(T=70, H=8200, E=4, k=1, I=64, E_local=1),
        dict(T=600, H=7168, E=4, k=2, I=64, E_local=2), dict(T=7, H=20000, E=8, k=8, I=64, E_local=6), dict(T=520, H=2504, E=32, k=32, I=64, E_local=32),
        dict(T=2100, H=4104, E=4, k=2, I=64, E_local=3)]


def layer_of(moe, d, seed):
    shapes = {"w_gate": (d.E_local, d.I, d.H), "w_up": (d.E_local, d.I, d.H), "w_down": (d.E_local, d.H, d.I)}
    if d.n_shared:
        shapes.update(sh_gate=(d.n_shared, d.I_shared, d.H), sh_up=(d.n_shared, d.I_shared, d.H), sh_down=(d.n_shared, d.H, d.I_shared))
    w = {n: randn(s, seed + i, 0.05) for i, (n, s) in enumerate(shapes.items())}
    local = None if d.E_local == d.E else torch.randperm(d.E, generator=gen(seed), device="cuda")[:d.E_local].to(torch.int32)
    return moe.MoeLayerF8(d, w, local)


def combined_exactly(moe, layer, logits, x):
    """The weighted sum of the layer's expert outputs in 64 bits, and what fp32 may
    leave of it: k + 1 additions of the terms' magnitudes."""
    d = layer.d
    rows, i32, bf = d.T * d.k, dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
    idx, gates = torch.empty((d.T, d.k), **i32), torch.empty((d.T, d.k), device="cuda")
    off, perm, inv = torch.empty(d.E_local + 1, **i32), torch.empty(rows, **i32), torch.empty((d.T, d.k), **i32)
    xp, yp = torch.empty((rows, d.H), **bf), torch.empty((rows, d.H), **bf)
    ysh = torch.empty((d.T, d.H), **bf) if d.n_shared else None
    moe.route(d, logits, idx, gates)
    moe.permute(d, idx, layer.local_experts, x, off, perm, inv, xp, moe.workspace(d, moe.ENTRY_PERMUTE))
    moe.expert_ffn_f8(d, xp, off, layer._w, x, yp, ysh, moe.workspace(d, moe.ENTRY_EXPERT_FFN_F8))
    y = torch.zeros((d.T, d.H), dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(y)
    for j in range(d.k):
        t = (inv[:, j] >= 0).nonzero().flatten()
        v = gates[t, j].double()[:, None] * yp[inv[t, j].long()].double()
        y[t] += v
        terms[t] += v.abs()
    if ysh is not None:
        y, terms = y + ysh.double(), terms + ysh.double().abs()
    return y, terms * (d.k + 2) * FP32


@pytest.mark.parametrize("case", range(len(ENDS)))
@pytest.mark.parametrize("post,gate,quant", [(False, "none", True), (True, "column", False), (True, "both", True)])
def test_layer_with_its_end(moe, case, post, gate, quant):
    """forward_f8 with norms: those of the weighted sum as it is in fp32; with `out`
    the layer's output too, bit for bit that of the layer without them."""
    d = moe.dims(S=1, **ENDS[case])
    layer = layer_of(moe, d, case)
    logits, x, h = torch.randn((d.T, d.E), generator=gen(case), device="cuda"), randn((d.T, d.H), 5), randn((d.T, d.H + 8), 6, 3.0)[:, :d.H]
    w, pw = randn((d.H,), 7), randn((d.H,), 8) if post else None
    g = None if GATES[gate] is None else randn(tuple(n if f else 1 for n, f in zip((d.T, d.H), GATES[gate])), 9)
    ho, xo = torch.empty((d.T, d.H), dtype=torch.bfloat16, device="cuda"), torch.empty((d.T, d.H), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((d.T, pad16(d.H)), dtype=torch.uint8, device="cuda").view(F8) if quant else None
    s = torch.empty((d.T, blocks(d.H)), device="cuda") if quant else None
    norm, io = moe.norm(d.H, w, pw, 0.875), moe.norm_io(h, ho, x=xo, q=q, scale=s, gate=g)
    plain = layer.forward(logits, None, x)
    assert layer.forward(logits, None, x, norm=norm, rows=io) is None
    y, ey = combined_exactly(moe, layer, logits, x)
    (rh, bh), (rx, bx, ex) = norm_and_bounds(y, h, pw, g, w, 0.875, 1e-6, 0.0)
    # what the sum's own rounding adds, through the norm of it (twice its share of the row's norm at most) and the gate
    r = 1.0 / torch.sqrt(y.square().mean(dim=1, keepdim=True) + 1e-6) * pw.double().abs() if post else torch.ones_like(y)
    z = y.abs() * r * (ey.square().sum(dim=1, keepdim=True) / (y.square().sum(dim=1, keepdim=True) + 1e-300)).sqrt() if post else 0.0
    more = 2.0 * (ey * r + z) * (1.0 if g is None else g.double().abs())
    within(ho, rh, bh + more * (1 + BF16))
    rr = 1.0 / torch.sqrt(rh.square().mean(dim=1, keepdim=True) + 1e-6)
    share = (more.square().sum(dim=1, keepdim=True) / rh.square().sum(dim=1, keepdim=True)).sqrt()
    mx = 2.0 * (more * rr * w.double().abs() + rx.abs() * share)
    within(xo, rx, bx + mx * (1 + BF16))
    if quant:
        assert_rows_of(q, s, rx, ex + mx)
    first, out = ho.clone(), torch.empty_like(plain)
    assert layer.forward(logits, None, x, out=out, norm=norm, rows=io) is out
    assert torch.equal(out, plain) and torch.equal(ho, first)


def test_blocks_in_a_row(moe):
    """Two layers as a model runs them: the first norm, the layer on the rows that it
    quantised, its end, the next layer on the rows of that; in a graph too.  The
    same by separate calls: every step's bf16 result, from the same inputs."""
    d = moe.dims(T=33, H=520, E=8, k=2, I=264, S=1, E_local=8, n_shared=1, I_shared=136)
    layers = [layer_of(moe, d, s) for s in (1, 20)]
    router = [torch.randn((d.H, d.E), generator=gen(s), device="cuda") for s in (3, 4)]
    h0 = randn((d.T, d.H), 6, 2.0)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    norms = [moe.norm(d.H, randn((d.H,), 30 + i), randn((d.H,), 40 + i) if i else None) for i in range(3)]
    q, s = torch.zeros((d.T, pad16(d.H)), dtype=torch.uint8, device="cuda").view(F8), torch.empty((d.T, blocks(d.H)), device="cuda")
    h, x, ws = torch.empty((d.T, d.H), **bf), torch.empty((d.T, d.H), **bf), moe.workspace(d, moe.ENTRY_FORWARD_F8)

    def fused():
        moe.norm_rows(norms[0], moe.norm_io(h0, h, x=x, q=q, scale=s))
        for i in range(2):
            layers[i].forward(x.float() @ router[i], None, xq=q, x_scale=s, norm=norms[i + 1], rows=moe.norm_io(h, h, x=x, q=q, scale=s), ws=ws)

    fused()
    torch.cuda.synchronize()
    got = h.clone(), x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fused()
    for _ in range(3):
        fused()
        torch.cuda.synchronize()
        assert torch.equal(h, got[0]) and torch.equal(x, got[1])
        h.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, got[0]) and torch.equal(x, got[1])
    # by separate calls: close (the layer's output is rounded between them, the rows
    # that a layer gets are quantised from fp32 in the one and from bf16 in the other)
    hs, xs = torch.empty((d.T, d.H), **bf), torch.empty((d.T, d.H), **bf)
    moe.norm_rows(norms[0], moe.norm_io(h0, hs, x=xs))
    logits = xs.float() @ router[0]
    y = layers[0].forward(logits, None, xs)
    moe.norm_rows(norms[1], moe.norm_io(hs, hs, x=xs), y=y)
    moe.norm_rows(norms[0], moe.norm_io(h0, h, x=x, q=q, scale=s))
    layers[0].forward(logits, None, xq=q, x_scale=s, norm=norms[1], rows=moe.norm_io(h, h, x=x), ws=ws)
    # e4m3's own error of a layer's output is 9 % of it at most (see test_gpu_f8.py); two roundings of x that differ
    # move it by far less, and the residual's rounding by 2^-8
    assert ((h.double() - hs.double()).norm() / hs.double().norm()).item() < 0.02
    assert ((x.double() - xs.double()).norm() / xs.double().norm()).item() < 0.02
