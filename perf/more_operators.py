"""The layer in 8-bit floating point and the norms around it, for timing and for comparing results.

A user who serves the layer from weights in e4m3, with one scale for each 128 x 128
block of a matrix and for each 128 columns of a token, calls:
  quantize   moe.quantize_rows_f8 for activations at every step, and
             moe.quantize_blocks_f8 for weights once;
  linear     moe.linear_f8: a dense product (projections around the layer, shared experts);
  grouped    moe.grouped_linear_f8: the same over ragged groups of rows, one weight
             matrix per expert, rows in place or read through a list;
  ffn        moe.expert_ffn_f8: the experts' SwiGLU networks on dispatched rows;
  norm       moe.norm_rows: the end of one block and the beginning of the next: the norm
             of what the block computed, its gate, the residual, and the next block's
             norm, whose rows may go out quantised;
  forward    moe.forward_f8: the whole layer of one step, with `norm` as its end.

The layers are those of paper_2606_15177_amd/workloads.py at the batch sizes that serving
meets, and generic ones that no tile divides.
"""
import math

import torch

own = False

# Layer shapes, by the workload they come from.
MIXTRAL = dict(H=4096, E=8, k=2, I=14336, E_local=8, n_shared=0, I_shared=0, zipf=1.0)
DSV2_LITE = dict(H=2048, E=64, k=6, I=1408, E_local=64, n_shared=2, I_shared=1408, zipf=1.0)
QWEN3 = dict(H=2048, E=128, k=8, I=768, E_local=128, n_shared=0, I_shared=0, zipf=0.6)
DSV3_SHARE = dict(H=7168, E=256, k=8, I=2048, E_local=32, n_shared=1, I_shared=2048, zipf=1.0)
RAGGED = dict(H=1000, E=24, k=3, I=520, E_local=10, n_shared=1, I_shared=344, zipf=0.8)

# How a block ends and the next one begins: `post` norms what the block computed, `gate`
# multiplies it (one value for each column, row or both), `pre` norms the sum for the next
# block, `quant` returns that norm's rows quantised too.
PLAIN_END = dict(post=False, gate="none", pre=True, rho=1.0)
FULL_END = dict(post=True, gate="column", pre=True, rho=0.875)


def listed():
    return [
        # a prefill batch on its way into the experts of an expert-parallel rank
        dict(name="quantize_rows_16384x7168", op="quantize", by="rows", G=1, M=16384, K=7168),
        # the experts of a layer as a program loads them, of sizes that no block divides
        dict(name="quantize_blocks_24x520x1000", op="quantize", by="blocks", G=24, M=520, K=1000),
        # one token through a shared expert's projection
        dict(name="linear_1x2048x7168", op="linear", M=1, N=2048, K=7168),
        # a prefill batch through gate and up of a shared expert as one matrix
        dict(name="linear_16384x4096x7168", op="linear", M=16384, N=4096, K=7168),
        # a decode batch over many small experts, its rows read through the dispatch list
        dict(name="grouped_256_qwen3_up", op="grouped", T=256, E=128, E_local=128, k=8, N=768, K=2048, gather=True, zipf=0.6),
        # a ragged chunk of sizes that no tile divides, fewer experts hosted here than routed
        dict(name="grouped_777_ragged", op="grouped", T=777, E=24, E_local=10, k=3, N=517, K=1003, gather=False, zipf=0.8),
        # a chunk of a chunked prefill mixed with decode tokens, shared experts beside the routed ones
        dict(DSV2_LITE, name="ffn_1021_dsv2_lite", op="ffn", T=1021),
        # a decode step of many users on few wide experts
        dict(MIXTRAL, name="ffn_64_mixtral", op="ffn", T=64),
        # one user's decode step between two blocks
        dict(FULL_END, name="norm_1x7168", op="norm", T=1, H=7168, pad=0, quant=True),
        # a prefill batch between two blocks, plain residual, rows of the stream lying apart
        dict(PLAIN_END, name="norm_16384x7168", op="norm", T=16384, H=7168, pad=64, quant=True),
        # one user's decode step: a single token through the layer and the norms after it
        dict(QWEN3, name="forward_1_qwen3", op="forward", T=1, quant=False, **FULL_END),
        # the largest: a prefill step of an expert-parallel rank
        dict(DSV3_SHARE, name="forward_16384_dsv3_share", op="forward", T=16384, quant=False, **PLAIN_END),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_end(rng, quant):
    return dict(post=rng.random() < 0.5, gate=rng.choice(["none", "column", "row", "both"]), pre=rng.random() < 0.85,
                quant=rng.random() < quant, rho=rng.choice([1.0, 0.875, round(rng.uniform(0.2, 1.0), 3)]))


def draw(rng):
    """One more case of the listed ranges: the named layers at other batch
    sizes, generic layers, products and rows of any sizes."""
    op = rng.choice(["quantize", "linear", "linear", "grouped", "ffn", "norm", "forward"])
    if op == "quantize":
        by = rng.choice(["rows", "blocks"])
        G = 1 if by == "rows" else rng.randint(1, 64)
        return dict(op=op, by=by, G=G, M=_log_int(rng, 1, 16384 // G), K=_log_int(rng, 64, 7168))
    if op == "linear":
        while True:
            c = dict(op=op, M=_log_int(rng, 1, 16384), N=_log_int(rng, 64, 14336), K=_log_int(rng, 64, 14336))
            if c["M"] * c["N"] * c["K"] <= 16384 * 4096 * 7168:
                return c
    if op == "grouped":
        E = rng.randint(4, 128)
        return dict(op=op, T=_log_int(rng, 1, 4096), E=E, E_local=rng.choice([E, rng.randint(max(1, E // 4), E)]),
                    k=rng.randint(1, min(8, E)), N=_log_int(rng, 64, 2048), K=_log_int(rng, 64, 2048),
                    gather=rng.random() < 0.5, zipf=round(rng.uniform(0.0, 1.2), 3))
    if op == "norm":
        return dict(_draw_end(rng, 0.6), op=op, T=_log_int(rng, 1, 16384), H=_log_int(rng, 64, 8192), pad=rng.choice([0, 0, 1, 64]))
    end = _draw_end(rng, 0.0) if op == "forward" else {}
    family = rng.choice(["mixtral", "dsv2", "qwen3", "dsv3", "generic", "generic"])
    if family == "mixtral":
        return dict(MIXTRAL, op=op, T=_log_int(rng, 1, 2000), **end)
    if family == "dsv2":
        return dict(DSV2_LITE, op=op, T=_log_int(rng, 1, 4096), **end)
    if family == "qwen3":
        return dict(QWEN3, op=op, T=_log_int(rng, 1, 8192), **end)
    if family == "dsv3":
        return dict(DSV3_SHARE, op=op, T=_log_int(rng, 8, 8192), **end)
    E = rng.randint(4, 96)
    n_shared = rng.randint(0, 2)
    return dict(op=op, T=_log_int(rng, 1, 3000), H=8 * rng.randint(8, 288), E=E, k=rng.randint(1, min(8, E)),
                I=8 * rng.randint(8, 192), E_local=rng.randint(max(1, E // 4), E), n_shared=n_shared,
                I_shared=8 * rng.randint(8, 192) if n_shared else 0, zipf=0.8, **end)


# ---- inputs ----

BLOCK = 128
EPS = 1e-6
F8 = torch.float8_e4m3fn


def _pad16(n):
    return (n + 15) // 16 * 16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _gen(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _acts(rows, cols, g):
    """Activations as after a norm: N(0, 1), one channel in a hundred eight
    times as large."""
    gain = 1.0 + 7.0 * (torch.rand((cols,), generator=g, device="cuda") < 0.01).float()
    return (torch.randn((rows, cols), generator=g, device="cuda") * gain).to(torch.bfloat16)


def _scaled(v, top):
    """v (32 bits) in steps of top / 448: the e4m3 values and the scale."""
    c448 = torch.full((), 448.0, device=v.device)
    return (v * 448.0 / torch.where(top > 0, top, torch.ones_like(top))).to(F8), top / c448


def _quantized(x):
    """e4m3 rows (padded with zeros to a multiple of 16) and a scale for each
    128 columns: scale = max|x| / 448, q = 448 x / max|x| to nearest, ties to even."""
    rows, cols = x.shape
    kb = _blocks(cols)
    q = torch.zeros((rows, _pad16(cols)), dtype=torch.uint8, device=x.device)
    scale = torch.zeros((rows, kb), dtype=torch.float32, device=x.device)
    step = max(1, (1 << 27) // cols)
    for a in range(0, rows, step):
        v = torch.nn.functional.pad(x[a:a + step].float(), (0, kb * BLOCK - cols)).view(-1, kb, BLOCK)
        f, s = _scaled(v, v.abs().amax(dim=2, keepdim=True))
        scale[a:a + step] = s[..., 0]
        q[a:a + step, :cols] = f.view(torch.uint8).view(-1, kb * BLOCK)[:, :cols]
    return q.view(F8), scale


def _quantized_blocks(x):
    """The same of matrices x [G, rows, cols] with a scale for each 128 x 128 block."""
    G, rows, cols = x.shape
    nb, kb = _blocks(rows), _blocks(cols)
    q = torch.zeros((G, rows, _pad16(cols)), dtype=torch.uint8, device=x.device)
    scale = torch.zeros((G, nb, kb), dtype=torch.float32, device=x.device)
    step = max(1, (1 << 27) // (rows * cols))
    for a in range(0, G, step):
        v = torch.nn.functional.pad(x[a:a + step].float(), (0, kb * BLOCK - cols, 0, nb * BLOCK - rows))
        v = v.view(-1, nb, BLOCK, kb, BLOCK)
        f, s = _scaled(v, v.abs().amax(dim=(2, 4), keepdim=True))
        scale[a:a + step] = s[:, :, 0, :, 0]
        q[a:a + step, :, :cols] = f.view(torch.uint8).view(-1, nb * BLOCK, kb * BLOCK)[:, :rows, :cols]
    return q.view(F8), scale


def _matrices(G, rows, cols, g):
    """bf16 matrices N(0, 0.02) whose rows differ in size."""
    w = torch.empty((G, rows, cols), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=g)
    return w * torch.exp(0.4 * torch.randn((G, rows, 1), generator=g, device="cuda")).to(torch.bfloat16)


def _weights(G, rows, cols, g):
    q = torch.empty((G, rows, _pad16(cols)), dtype=torch.uint8, device="cuda")
    scale = torch.empty((G, _blocks(rows), _blocks(cols)), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 28) // (rows * cols))
    for a in range(0, G, step):
        n = min(step, G - a)
        f, scale[a:a + n] = _quantized_blocks(_matrices(n, rows, cols, g))
        q[a:a + n] = f.view(torch.uint8)
    return q.view(F8), scale


def _sizes(case, g):
    """Rows of each hosted expert (host list), of T k pairs routed by a Zipf popularity."""
    p = (1.0 + torch.randperm(case["E"], generator=g).double()) ** -case["zipf"]
    T, k = case["T"], case["k"]
    ids = torch.multinomial(p.repeat(T, 1), k, generator=g) if k < case["E"] else torch.arange(case["E"]).repeat(T, 1)
    rows = torch.bincount(ids.reshape(-1), minlength=case["E"])
    return rows[:case["E_local"]].tolist()


def _offsets(sizes):
    o = [0]
    for n in sizes:
        o.append(o[-1] + n)
    return o


def _layer_weights(case, g):
    EL, H, I = case["E_local"], case["H"], case["I"]
    w = {}
    for n, rows, cols in (("gate", I, H), ("up", I, H), ("down", H, I)):
        w["w_" + n], w["s_" + n] = _weights(EL, rows, cols, g)
    if case["n_shared"]:
        width = case["n_shared"] * case["I_shared"]
        for n, rows, cols in (("gate", width, H), ("up", width, H), ("down", H, width)):
            q, s = _weights(1, rows, cols, g)
            w["sh_" + n], w["sh_s_" + n] = q[0], s[0]
    return w


def _end_inputs(case, g):
    """The residual stream and what the norms hold."""
    T, H = case["T"], case["H"]
    s = dict(h=(4.0 * torch.randn((T, H + case.get("pad", 0)), generator=g, device="cuda")).to(torch.bfloat16)[:, :H])

    def vector(*shape):
        return (1.0 + 0.3 * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)

    s["post_weight"] = vector(H) if case["post"] else None
    s["weight"] = vector(H) if case["pre"] else None
    s["gate"] = None if case["gate"] == "none" else vector(*{"column": (1, H), "row": (T, 1), "both": (T, H)}[case["gate"]])
    return s


def _inputs(case, seed):
    g, gc = _gen(seed, "cuda"), _gen(seed, "cpu")
    op = case["op"]
    if op == "quantize":
        if case["by"] == "rows":
            return dict(x=_acts(case["M"], case["K"], g))
        return dict(x=_matrices(case["G"], case["M"], case["K"], g))
    if op == "linear":
        s = dict(zip(("xq", "xs"), _quantized(_acts(case["M"], case["K"], g))))
        q, sc = _weights(1, case["N"], case["K"], g)
        s["wq"], s["ws"] = q[0], sc[0]
        return s
    if op == "grouped":
        sizes = _sizes(case, gc)
        R, M = sum(sizes), case["T"] * case["k"]
        s = dict(sizes=sizes, offsets=torch.tensor(_offsets(sizes), dtype=torch.int32, device="cuda"))
        s["xq"], s["xs"] = _quantized(_acts(case["T"] if case["gather"] else M, case["K"], g))
        # tokens ascend within a group, as a dispatch leaves them
        s["x_rows"] = None
        if case["gather"]:
            rows = [torch.sort(torch.randperm(case["T"], generator=gc)[:n]).values for n in sizes]
            rows.append(torch.zeros((M - R,), dtype=torch.int64))
            s["x_rows"] = torch.cat(rows).to(torch.int32).cuda()
        s["wq"], s["ws"] = _weights(case["E_local"], case["N"], case["K"], g)
        return s
    if op == "norm":
        return dict(_end_inputs(case, g), y=_acts(case["T"], case["H"], g))
    s = dict(w=_layer_weights(case, g))
    if op == "ffn":
        s["sizes"] = _sizes(case, gc)
        s["offsets"] = torch.tensor(_offsets(s["sizes"]), dtype=torch.int32, device="cuda")
        s["x_perm"] = _acts(case["T"] * case["k"], case["H"], g)
        s["x"] = _acts(case["T"], case["H"], g) if case["n_shared"] else None
        return s
    rank = 1.0 + torch.randperm(case["E"], generator=g, device="cuda").float()
    s["logits"] = torch.randn((case["T"], case["E"]), generator=g, device="cuda") - case["zipf"] * torch.log(rank)
    s["local"] = None
    if case["E_local"] < case["E"]:
        s["local"] = torch.randperm(case["E"], generator=g, device="cuda")[:case["E_local"]].to(torch.int32)
    s["x"] = _acts(case["T"], case["H"], g)
    s.update(_end_inputs(case, g))
    # the norm before the layer leaves its rows quantised
    s["xq"], s["xs"] = _quantized(s["x"])
    return s


def _dims(case):
    from paper_2606_15177_amd import moe
    return moe.dims(case["T"], case["H"], case["E"], case["k"], case["I"], 1, case["E_local"], case["n_shared"], case["I_shared"])


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]

    def zeros(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    if op == "quantize":
        G, M, K = case["G"], case["M"], case["K"]
        if case["by"] == "rows":
            s["q"], s["scale"] = zeros(M, _pad16(K), dtype=torch.uint8).view(F8), zeros(M, _blocks(K), dtype=torch.float32)
        else:
            s["q"], s["scale"] = zeros(G, M, _pad16(K), dtype=torch.uint8).view(F8), zeros(G, _blocks(M), _blocks(K), dtype=torch.float32)
    elif op == "linear":
        s["out"] = zeros(case["M"], case["N"])
    elif op == "grouped":
        s["out"] = zeros(case["T"] * case["k"], case["N"])
    elif op == "ffn":
        s["out"] = zeros(case["T"] * case["k"], case["H"])
        s["out_shared"] = zeros(case["T"], case["H"]) if case["n_shared"] else None
    else:
        T, H = case["T"], case["H"]
        s["h_out"] = zeros(T, H)
        s["x_out"] = zeros(T, H) if case["pre"] else None
        s["q"] = zeros(T, _pad16(H), dtype=torch.uint8).view(F8) if case["pre"] and case["quant"] else None
        s["scale"] = zeros(T, _blocks(H), dtype=torch.float32) if case["pre"] and case["quant"] else None
        if own:
            from paper_2606_15177_amd import moe
            s["norm"] = moe.norm(H, weight=s["weight"], post_weight=s["post_weight"], residual_scale=case["rho"], eps=EPS)
    if own and op in ("ffn", "forward"):
        from paper_2606_15177_amd import moe
        s["d"] = _dims(case)
        s["handle"] = moe.make_weights_f8(s["d"], s["w"])
        s["work"] = moe.workspace(s["d"], moe.ENTRY_EXPERT_FFN_F8 if op == "ffn" else moe.ENTRY_FORWARD_F8)
    return s


# ---- the plain forms ----


def _values(q, s, K):
    """The values that rows and their scales stand for, in 32 bits."""
    return q[..., :K].float() * torch.repeat_interleave(s, BLOCK, dim=-1)[..., :K]


def _matrix(q, s, N, K):
    return q[..., :K].float() * torch.repeat_interleave(torch.repeat_interleave(s, BLOCK, dim=-2)[..., :N, :], BLOCK, dim=-1)[..., :K]


def _swiglu(x, w, p, sl, H, I):
    """The SwiGLU network of rows x (32 bits, quantised); its hidden rows are
    held in bf16 and quantised like the inputs."""
    gate = x @ _matrix(w[p[0] + "gate"][sl], w[p[1] + "gate"][sl], I, H).t()
    up = x @ _matrix(w[p[0] + "up"][sl], w[p[1] + "up"][sl], I, H).t()
    hidden = _values(*_quantized((gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)), I)
    return hidden @ _matrix(w[p[0] + "down"][sl], w[p[1] + "down"][sl], H, I).t()


def _rms(v, weight):
    return v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + EPS) * weight.float()


def _end(s, y):
    """The end of the block that computed y (32 bits), and the next one's beginning;
    each output is rounded once."""
    case = s["case"]
    z = _rms(y, s["post_weight"]) if case["post"] else y
    if s["gate"] is not None:
        z = z * s["gate"].float()
    h = case["rho"] * s["h"].float() + z
    out = dict(h=h.to(torch.bfloat16))
    if case["pre"]:
        x = _rms(h, s["weight"])
        out["x"] = x.to(torch.bfloat16)
        if case["quant"]:
            out["q"], out["scale"] = _quantized(x)
    return out


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        return dict(zip(("q", "scale"), (_quantized if case["by"] == "rows" else _quantized_blocks)(s["x"])))
    if op == "linear":
        w = _matrix(s["wq"], s["ws"], case["N"], case["K"])
        return (_values(s["xq"], s["xs"], case["K"]) @ w.t()).to(torch.bfloat16)
    if op == "norm":
        return _end(s, s["y"].float())
    if op == "grouped":
        N, K = case["N"], case["K"]
        y = torch.zeros((case["T"] * case["k"], N), dtype=torch.bfloat16, device="cuda")
        x = _values(s["xq"], s["xs"], K)
        a = 0
        for e, n in enumerate(s["sizes"]):
            if n:
                rows = s["x_rows"][a:a + n].long() if s["x_rows"] is not None else slice(a, a + n)
                y[a:a + n] = (x[rows] @ _matrix(s["wq"][e], s["ws"][e], N, K).t()).to(torch.bfloat16)
            a += n
        return y
    H, I, w = case["H"], case["I"], s["w"]
    width = case["n_shared"] * case["I_shared"]
    if op == "ffn":
        shared = None
        if width:
            shared = _swiglu(_values(*_quantized(s["x"]), H), w, ("sh_", "sh_s_"), slice(None), H, width).to(torch.bfloat16)
        y = torch.zeros((case["T"] * case["k"], H), dtype=torch.bfloat16, device="cuda")
        x = _values(*_quantized(s["x_perm"]), H)
        a = 0
        for e, n in enumerate(s["sizes"]):
            if n:
                y[a:a + n] = _swiglu(x[a:a + n], w, ("w_", "s_"), e, H, I).to(torch.bfloat16)
            a += n
        return dict(y=y, y_shared=shared)
    x = _values(s["xq"], s["xs"], H)
    # equal logits to the lower expert
    top, idx = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    top, idx = top[:, :case["k"]], idx[:, :case["k"]]
    gates = torch.exp(top - top[:, :1])
    gates = gates / gates.sum(dim=1, keepdim=True)
    y = _swiglu(x, w, ("sh_", "sh_s_"), slice(None), H, width) if width else torch.zeros_like(x)
    for slot, e in enumerate(range(case["E"]) if s["local"] is None else s["local"].tolist()):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        if len(t):
            y.index_add_(0, t, gates[t, j][:, None] * _swiglu(x[t], w, ("w_", "s_"), slot, H, I))
    return _end(s, y)


def run(state):
    if not own:
        return _plain(state)
    from paper_2606_15177_amd import moe
    s, case = state, state["case"]
    op = case["op"]
    if op == "quantize":
        (moe.quantize_rows_f8 if case["by"] == "rows" else moe.quantize_blocks_f8)(s["x"], s["q"], s["scale"])
        return dict(q=s["q"], scale=s["scale"])
    if op == "linear":
        moe.linear_f8(case["K"], s["xq"], s["xs"], s["wq"], s["ws"], s["out"])
        return s["out"]
    if op == "grouped":
        moe.grouped_linear_f8(case["K"], s["xq"], s["xs"], s["offsets"], s["wq"], s["ws"], s["out"], x_rows=s["x_rows"])
        return s["out"]
    if op == "ffn":
        moe.expert_ffn_f8(s["d"], s["x_perm"], s["offsets"], s["handle"], s["x"], s["out"], s["out_shared"], s["work"])
        return dict(y=s["out"], y_shared=s["out_shared"])
    rows = moe.norm_io(s["h"], s["h_out"], x=s["x_out"], q=s["q"], scale=s["scale"], gate=s["gate"])
    if op == "norm":
        moe.norm_rows(s["norm"], rows, y=s["y"])
    else:
        moe.forward_f8(s["d"], s["logits"], None, None, s["local"], s["handle"], None, None, s["work"], xq=s["xq"], x_scale=s["xs"],
                       norm=s["norm"], rows=rows)
    out = dict(h=s["h_out"])
    if case["pre"]:
        out["x"] = s["x_out"]
        if case["quant"]:
            out["q"], out["scale"] = s["q"], s["scale"]
    return out


# ---- what a pass cannot do without ----


def _end_work(case):
    """Bytes of the residual read and written, and of the next block's rows."""
    n = case["T"] * case["H"]
    rows = 2 * n * case["pre"] + (n + 4 * case["T"] * _blocks(case["H"])) * (case["pre"] and case["quant"])
    return 4 * n + rows + 2 * n * (case["gate"] == "both")


def work(case):
    op = case["op"]
    if op == "quantize":
        G, M, K = case["G"], case["M"], case["K"]
        scales = M * _blocks(K) if case["by"] == "rows" else G * _blocks(M) * _blocks(K)
        return {"bytes": G * M * (2 * K + _pad16(K)) + 4 * scales, "flops": 3 * G * M * K}
    if op == "norm":
        n = case["T"] * case["H"]
        return {"bytes": 2 * n + _end_work(case), "flops": n * (3 + 4 * case["post"] + (case["gate"] != "none") + 4 * case["pre"])}

    def matrix(N, K):
        return N * K + 4 * _blocks(N) * _blocks(K)

    def rows(M, K):
        return M * (K + 4 * _blocks(K))

    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": rows(M, K) + matrix(N, K) + 2 * M * N, "flops": 2 * M * N * K}
    sizes = _sizes(case, _gen(0, "cpu"))
    R, active = sum(sizes), sum(n > 0 for n in sizes)
    if op == "grouped":
        N, K = case["N"], case["K"]
        x = min(R, case["T"]) if case["gather"] else R
        return {"bytes": rows(x, K) + active * matrix(N, K) + 2 * R * N, "flops": 2 * R * N * K}
    H, I, T = case["H"], case["I"], case["T"]
    width = case["n_shared"] * case["I_shared"]
    weights = active * (2 * matrix(I, H) + matrix(H, I)) + (2 * matrix(width, H) + matrix(H, width) if width else 0)
    flops = 6 * H * (I * R + width * T)
    if op == "ffn":
        return {"bytes": weights + 2 * R * H * 2 + (2 * T * H * 2 if width else 0), "flops": flops}
    return {"bytes": weights + rows(T, H) + T * case["E"] * 4 + _end_work(case), "flops": flops}


# ---- the same in 64 bits, from the definitions ----


def _e4m3(v):
    """v (64 bits, up to 448) to the nearest e4m3 value, ties to even: four
    significant bits, steps of 2^-9 at least."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(v.abs(), min=1e-30))), min=-6.0) - 3.0)
    return torch.round(v / step) * step


def _spread(s, n, dim):
    """Scales by column (or row): one of each block for its members."""
    return s.double().index_select(dim, torch.arange(n, device=s.device) // BLOCK)


def _rows64(v):
    """e4m3 values and scales of the rows of v (64 bits)."""
    n, m = v.shape
    top = torch.stack([c.abs().max(dim=1).values for c in v.split(BLOCK, dim=1)], dim=1)
    at = _spread(top, m, 1)
    return torch.where(at > 0, _e4m3(448.0 * v / torch.where(at > 0, at, 1.0)), 0.0), top / 448.0


def _through_rows64(v):
    q, s = _rows64(v)
    return q * _spread(s, v.shape[1], 1)


def _norm64(v, weight):
    return weight.double() * v * torch.rsqrt(v.square().sum(dim=1, keepdim=True) / v.shape[1] + EPS)


def _end64(case, s, y):
    z = _norm64(y, s["post_weight"]) if case["post"] else y
    z = z if s["gate"] is None else s["gate"].double() * z
    h = z + s["h"].double() * case["rho"]
    out = dict(h=h)
    if case["pre"]:
        out["x"] = _norm64(h, s["weight"])
        if case["quant"]:
            q, out["scale"] = _rows64(out["x"])
            out["q"] = torch.zeros((q.shape[0], _pad16(case["H"])), dtype=torch.float64, device="cuda")
            out["q"][:, :case["H"]] = q
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        x = s["x"].double()
        if case["by"] == "rows":
            q, scale = _rows64(x)
        else:
            G, M, K = x.shape
            scale = torch.zeros((G, _blocks(M), _blocks(K)), dtype=torch.float64, device="cuda")
            q = torch.zeros_like(x)
            for i in range(_blocks(M)):
                for j in range(_blocks(K)):
                    at = (slice(None), slice(BLOCK * i, BLOCK * (i + 1)), slice(BLOCK * j, BLOCK * (j + 1)))
                    top = x[at].abs().flatten(1).max(dim=1).values
                    scale[:, i, j] = top / 448.0
                    q[at] = _e4m3(448.0 * x[at] / torch.where(top > 0, top, 1.0)[:, None, None])
        full = torch.zeros(tuple(x.shape[:-1]) + (_pad16(case["K"]),), dtype=torch.float64, device="cuda")
        full[..., :case["K"]] = q
        return dict(q=full, scale=scale)
    if op == "norm":
        return _end64(case, s, s["y"].double())

    def deq(q, sc, N, K):
        return q[:, :K].double() * _spread(_spread(sc, N, 0), K, 1)

    if op in ("linear", "grouped"):
        N, K = case["N"], case["K"]
        x = s["xq"][:, :K].double() * _spread(s["xs"], K, 1)
        if op == "linear":
            return x @ deq(s["wq"], s["ws"], N, K).t()
        y = torch.zeros((case["T"] * case["k"], N), dtype=torch.float64, device="cuda")
        for e in range(case["E_local"]):
            a, b = int(s["offsets"][e]), int(s["offsets"][e + 1])
            if a < b:
                rows = x[a:b] if s["x_rows"] is None else x.index_select(0, s["x_rows"][a:b].long())
                y[a:b] = rows @ deq(s["wq"][e], s["ws"][e], N, K).t()
        return y
    H, I, w, width = case["H"], case["I"], s["w"], case["n_shared"] * case["I_shared"]

    def network(x, p, ps, e, n):
        """x in 64 bits, quantised; the hidden rows have the values that bf16 holds."""
        g, u = (x @ deq(w[p + m][e], w[ps + m][e], n, H).t() for m in ("gate", "up"))
        hidden = _through_rows64((torch.sigmoid(g) * g * u).to(torch.bfloat16).double())
        return hidden @ deq(w[p + "down"][e], w[ps + "down"][e], H, n).t()

    x = _through_rows64(s["x"].double()) if s["x"] is not None else None
    shared = network(x, "sh_", "sh_s_", slice(None), width) if width else None
    if op == "ffn":
        y = torch.zeros((case["T"] * case["k"], H), dtype=torch.float64, device="cuda")
        a = 0
        for e, n in enumerate(s["sizes"]):
            y[a:a + n] = network(_through_rows64(s["x_perm"][a:a + n].double()), "w_", "s_", e, I) if n else 0.0
            a += n
        return dict(y=y, y_shared=shared)
    lg = s["logits"].double()
    idx = torch.argsort(lg, dim=1, descending=True, stable=True)[:, :case["k"]]
    gates = torch.zeros_like(lg).scatter_(1, idx, torch.softmax(lg.gather(1, idx), dim=1))
    out = torch.zeros((case["T"], H), dtype=torch.float64, device="cuda") if shared is None else shared
    hosted = list(range(case["E"])) if s["local"] is None else s["local"].tolist()
    for slot, e in enumerate(hosted):
        t = torch.nonzero(gates[:, e] > 0).flatten()
        if t.numel():
            out[t] += gates[t, e].unsqueeze(1) * network(x[t], "w_", "s_", slot, I)
    return _end64(case, s, out)
