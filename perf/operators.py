"""Operators beside the pruned layer, as users of the library call them: what they have in hand, one pass, and what the pass
cannot do without.  `run` computes them in their plain form, or with `own` through the library.

Five paths, each over the range of sizes that it meets (`draw` gives more cases of the same ranges):

  layer8     Y = act(X W^T + bias) + residual with X and W in 8-bit floating point (e4m3), X with a scale for every 128 columns of
             a row, W (the masked dense matrix, in 8 bits once per model) for every 128 x 128 block; all scales are powers of two
  train8     the three products of a layer in training, everything brought to 8 bits in the step: Y, dX = dY W (its sums along the
             outputs) and dW = dY^T X (along the tokens, in fp32)
  join       after a block and before the next: Z = x_scale X + gate * N(F), H = N(Z); each norm and the gate may be absent
  join_back  its gradients, from what a program keeps of the forward pass
  adamw      one decoupled-decay Adam step over all tensors of a model, moments in 32 bits or in 8

Matrices are BERT-like (hidden h: 3h x h, h x h, 4h x h, h x 4h) and larger ones of the same kind; weights N(0, 0.02),
activations N(0, 1) with a few columns ten times as large, gradients small.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_E4M3 = torch.float8_e4m3fn
_LAYER, _RMS = "layer", "rms"


def listed():
    return [
        # one token at a server: the weights are read once and little is computed
        dict(name="layer8_token", path="layer8", T=1, M=4096, N=1024, dtype="bf16", bias=True, gelu=True, residual=False),
        # a short ragged request through matrices whose sides are no multiples of anything
        dict(name="layer8_ragged", path="layer8", T=333, M=1111, N=690, dtype="f16", bias=True, gelu=False, residual=True),
        # the benchmark's batch (64 sequences of 128 tokens) through the FFN up-projection
        dict(name="layer8_batch", path="layer8", T=8192, M=4096, N=1024, dtype="bf16", bias=True, gelu=True, residual=False),
        # a long prompt through a wide layer: the matrix cores
        dict(name="layer8_wide", path="layer8", T=16384, M=4096, N=4096, dtype="bf16", bias=False, gelu=False, residual=False),
        # a training step of the FFN down-projection
        dict(name="train8_batch", path="train8", T=8192, M=1024, N=4096, dtype="bf16"),
        # one token after a block: BERT's form (norm after the addition)
        dict(name="join_token", path="join", T=1, H=1024, dtype="bf16", kind=_LAYER, post=False, pre=True, gate=0, x_scale=1.0),
        # a batch with a norm on either side of the block and a learned gate per channel
        dict(name="join_batch", path="join", T=8192, H=1024, dtype="bf16", kind=_RMS, post=True, pre=True, gate=1, x_scale=1.0),
        # the batch's backward pass in BERT's form
        dict(name="join_back_batch", path="join_back", T=8192, H=1024, dtype="bf16", kind=_LAYER, post=False, pre=True, gate=0, x_scale=1.0),
        # both norms, a gate per sequence, an odd width in single precision
        dict(name="join_back_odd", path="join_back", T=1536, H=770, dtype="f32", kind=_LAYER, post=True, pre=True, gate=12, x_scale=0.81),
        # one encoder layer of a small model, as it is fine-tuned: latency
        dict(name="adamw_small", path="adamw", layers=1, hidden=250, bits=32, grad="f32", masked=False),
        # all tensors of a 24-layer model with their masks, moments in single precision
        dict(name="adamw_model", path="adamw", layers=24, hidden=1024, bits=32, grad="bf16", masked=True),
        # the same model, moments in 8 bits
        dict(name="adamw_model8", path="adamw", layers=24, hidden=1024, bits=8, grad="bf16", masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    path = rng.choice(("layer8", "layer8", "train8", "join", "join_back", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if path == "layer8":
        M, N = _log(rng, 64, 8192), _log(rng, 64, 8192)
        T = _log(rng, 1, min(16384, (16384 * 4096 * 4096) // (M * N)))
        return dict(path=path, T=T, M=M, N=N, dtype=dtype, bias=rng.random() < 0.7, gelu=rng.random() < 0.3, residual=rng.random() < 0.3)
    if path == "train8":
        M, N = _log(rng, 64, 4096), _log(rng, 64, 4096)
        return dict(path=path, T=_log(rng, 32, min(16384, (3 * 8192 * 4096 * 1024) // (M * N))), M=M, N=N, dtype=dtype)
    if path in ("join", "join_back"):
        H = _log(rng, 64, 8192)
        groups = rng.choice((0, 0, 1, 1, rng.randint(2, 32)))
        T = _log(rng, 1, min(32768, 8192 * 1024 // H))
        if groups > 1:
            T = (T + groups - 1) // groups * groups
        post = rng.random() < 0.5
        return dict(path=path, T=T, H=H, dtype=dtype, kind=rng.choice((_LAYER, _RMS)), post=post, pre=not post or rng.random() < 0.7,
                    gate=groups, x_scale=rng.choice((1.0, 1.0, 0.81)))
    return dict(path=path, layers=rng.randint(1, 12), hidden=_log(rng, 64, 1024), bits=rng.choice((32, 8)), grad=rng.choice(("f32", "bf16")),
                masked=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _activations(gen, T, N, dtype):
    x = torch.empty((T, N), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen)
    x[:, torch.randint(0, N, (max(1, N // 100),), generator=gen, device="cuda")] *= 10.0
    return x.to(dtype)


def _blocks_up(x, dim):
    """x, zeros behind it up to whole blocks of 128 along dim."""
    more = -x.shape[dim] % 128
    if not more:
        return x
    shape = list(x.shape)
    shape[dim] = more
    return torch.cat([x, torch.zeros(shape, dtype=x.dtype, device=x.device)], dim)


def _exponents(largest):
    """The least e with largest / 2^e <= 448, held in 8 bits with a bias of 127; 127 for zero."""
    f, k = torch.frexp(largest)  # largest = f 2^k, f in [0.5, 1); 448 = 0.875 2^9
    e = k - 9 + (f > 0.875).to(k.dtype)
    return torch.where(largest > 0, e.clamp(-127, 127) + 127, torch.full_like(e, 127)).to(torch.int32)


def _power(e):
    """2^(e - 127) for whole numbers e of 0 to 254, exactly."""
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _to8(x, block):
    """The codes of x [rows, columns padded to 128] and the biased exponents of its scales: per row and 128 columns, or (block) per
    128 x 128 block."""
    rows = x.shape[0]
    x = _blocks_up(x, 1)
    if block:
        x = _blocks_up(x, 0)
    y = x.view(-1, 128 if block else 1, x.shape[1] // 128, 128)
    e = _exponents(y.abs().amax(dim=(1, 3)))
    codes = (y * _power(254 - e)[:, None, :, None]).to(_E4M3).view(x.shape)
    return codes[:rows], e


def _from8(codes, e, block):
    """The matrix that codes and scales stand for, in single precision."""
    e = e.to(torch.int32)
    if block:
        e = e.repeat_interleave(128, 0)[:codes.shape[0]]
    return (codes.float().view(codes.shape[0], -1, 128) * _power(e)[:, :, None]).view(codes.shape)


def _tensors(case):
    """Rows, columns and decay of every tensor of the model: per layer four matrices, their biases and two norms."""
    h = case["hidden"]
    layer = []
    for M, N in ((3 * h, h), (h, h), (4 * h, h), (h, 4 * h)):
        layer += [(M, N, 0.01), (1, M, 0.0)]
    return (layer + 4 * [(1, h, 0.0)]) * case["layers"]


def _rows(case, M):
    """Rows of a row-block of the masks."""
    return 16 if M % 16 == 0 else 2 if M % 2 == 0 else 1


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    path = case["path"]
    s = dict(case=case)
    if path == "adamw":
        shapes = _tensors(case)
        n = sum(M * N for M, N, _ in shapes)
        eight = case["bits"] == 8
        s["w"], s["g"] = _normal(gen, (n,), 0.02, torch.float32), _normal(gen, (n,), 1e-3, _DT[case["grad"]])
        s["copy"] = s["w"].bfloat16()
        if eight:  # the moments: codes, and per tensor two rows of scales, one for every 256 elements
            blocks = sum((M * N + 255) // 256 for M, N, _ in shapes)
            s["m"] = _normal(gen, (n,), 120.0, torch.float32).clamp_(-448, 448).to(_E4M3)
            s["v"] = _normal(gen, (n,), 120.0, torch.float32).abs_().clamp_(2.0 ** -9, 448).to(_E4M3)
            s["scales"] = torch.empty(2 * blocks, device="cuda").uniform_(0.5e-6, 2e-6, generator=gen)
        else:
            s["m"], s["v"] = _normal(gen, (n,), 3e-4, torch.float32), _normal(gen, (n,), 1e-3, torch.float32).square_()
        s["lists"] = {k: [] for k in ("w", "g", "copy", "m", "v", "scales", "keep")}
        at = blk = 0
        for M, N, _ in shapes:
            for k in ("w", "g", "copy", "m", "v"):
                s["lists"][k].append(s[k][at:at + M * N].view(M, N))
            at += M * N
            nb = (M * N + 255) // 256
            if eight:
                s["lists"]["scales"].append(s["scales"][2 * blk:2 * (blk + nb)].view(2, nb))
            blk += nb
            masked = case["masked"] and M > 1
            s["lists"]["keep"].append((torch.rand((M // _rows(case, M), N), generator=gen, device="cuda") < 0.5).to(torch.uint8) if masked else None)
        s["decay"] = [d for _, _, d in shapes]
        s["rows"] = [_rows(case, M) for M, _, _ in shapes]
        return s
    dt, T = _DT[case["dtype"]], case["T"]
    if path == "layer8":
        M, N = case["M"], case["N"]
        s["x"] = _activations(gen, T, N, dt)
        codes, e = _to8(_normal(gen, (M, N), 0.02, dt).float(), True)
        s["w"] = (codes, e.to(torch.uint8))
        s["bias"] = _normal(gen, (M,), 0.02, dt) if case["bias"] else None
        s["residual"] = _normal(gen, (T, M), 1.0, dt) if case["residual"] else None
    elif path == "train8":
        M, N = case["M"], case["N"]
        s["x"], s["dy"], s["w"] = _activations(gen, T, N, dt), _normal(gen, (T, M), 1e-3, dt), _normal(gen, (M, N), 0.02, dt)
    else:
        H = case["H"]
        s["x"], s["f"] = _activations(gen, T, H, dt), _normal(gen, (T, H), 0.5, dt)
        s["gate"] = _normal(gen, (case["gate"], H), 0.5, dt) if case["gate"] else None
        for n in ("post", "pre"):
            s["w_" + n] = (1.0 + _normal(gen, (H,), 0.1, torch.float32)).to(dt) if case[n] else None
            s["b_" + n] = _normal(gen, (H,), 0.1, dt) if case[n] and case["kind"] == _LAYER else None
        if path == "join_back":  # what the forward pass leaves: the sum, and mean and 1 / deviation of every row
            s["dz"], s["dh"] = _normal(gen, (T, H), 1e-2, dt), _normal(gen, (T, H), 1e-2, dt) if case["pre"] else None
            f = s["f"].float()
            s["stats_post"] = _stats(case, f) if case["post"] else None
            if case["post"]:
                f = _affine(_normed(f, s["stats_post"]), s["w_post"], s["b_post"])
            if case["gate"]:
                f = f * _per_row(s["gate"], T)
            s["z"] = (case["x_scale"] * s["x"].float() + f).to(dt) if case["pre"] else None
            s["stats_pre"] = _stats(case, s["z"].float()) if case["pre"] else None
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------------------
_EPS = 1e-6


def _stats(case, x):
    """Mean (0 for the root mean square) and 1 / deviation of every row: [rows, 2]."""
    mean = x.mean(1, keepdim=True) if case["kind"] == _LAYER else torch.zeros_like(x[:, :1])
    return torch.cat([mean, 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + _EPS)], 1)


def _normed(x, stats):
    return (x - stats[:, :1]) * stats[:, 1:]


def _affine(x, w, b):
    return x * w.to(x.dtype) + (0 if b is None else b.to(x.dtype))


def _per_row(gate, T):
    return gate.repeat_interleave(T // gate.shape[0], 0)


def _layer8(s):
    case = s["case"]
    xc, xe = _to8(s["x"].float(), False)
    y = torch.matmul(_from8(xc, xe, False), _from8(*s["w"], True).t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["gelu"]:
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _train8(s):
    T, M, N = (s["case"][k] for k in "TMN")
    x, dy, w = s["x"].float(), s["dy"].float(), s["w"].float()
    of = lambda m, block=False: _from8(*_to8(m.contiguous(), block), block)  # noqa: E731
    w8 = of(w, True)
    y = torch.matmul(of(x), w8.t())
    dx = torch.matmul(of(dy)[:, :M], w8[:, :N])
    dw = torch.matmul(of(dy.t()), of(x.t()).t())
    return {"y": y.to(s["x"].dtype), "dx": dx.to(s["x"].dtype), "dw": dw}


def _join(s):
    case, dt = s["case"], s["x"].dtype
    f = s["f"].float()
    out = {}
    if case["post"]:
        out["stats_post"] = _stats(case, f)
        f = _affine(_normed(f, out["stats_post"]), s["w_post"], s["b_post"])
    if case["gate"]:
        f = f * _per_row(s["gate"].float(), case["T"])
    out["z"] = (case["x_scale"] * s["x"].float() + f).to(dt)
    if case["pre"]:  # of the sum as it is stored
        z = out["z"].float()
        out["stats_pre"] = _stats(case, z)
        out["h"] = _affine(_normed(z, out["stats_pre"]), s["w_pre"], s["b_pre"]).to(dt)
    return out


def _norm_back(case, dy, x, stats, w):
    """Gradients of the norm's input (without what dy has besides), its weight and its bias."""
    hat, g = _normed(x, stats), dy * w.to(dy.dtype)
    dx = g - hat * (g * hat).mean(1, keepdim=True)
    if case["kind"] == _LAYER:
        dx = dx - g.mean(1, keepdim=True)
    return dx * stats[:, 1:], (dy * hat).sum(0), dy.sum(0) if case["kind"] == _LAYER else None


def _join_back(s):
    case, T = s["case"], s["case"]["T"]
    to = lambda t: None if t is None else t.float()  # noqa: E731
    out, dz = {}, to(s["dz"])
    if case["pre"]:
        d, out["dw_pre"], out["db_pre"] = _norm_back(case, to(s["dh"]), to(s["z"]), to(s["stats_pre"]), to(s["w_pre"]))
        dz = dz + d
    out["dx"] = case["x_scale"] * dz
    n, df = to(s["f"]), dz
    if case["post"]:
        n = _affine(_normed(n, to(s["stats_post"])), s["w_post"], s["b_post"])
    if case["gate"]:
        out["dgate"] = (dz * n).view(case["gate"], -1, case["H"]).sum(1)
        df = dz * _per_row(to(s["gate"]), T)
    if case["post"]:
        df, out["dw_post"], out["db_post"] = _norm_back(case, df, to(s["f"]), to(s["stats_post"]), to(s["w_post"]))
    out["df"] = df
    return {k: v.to(s["dz"].dtype) if k in ("dx", "df") else v for k, v in out.items() if v is not None}


_BETA1, _BETA2, _ADAM_EPS, _LR, _STEP, _SEED = 0.9, 0.999, 1e-8, 1e-4, 10, 1234


def _bits(index, step, seed):
    """32 mixed bits of an element's place in its tensor, the step and the seed, as 64-bit whole numbers."""
    low = 0xFFFFFFFF
    x = (index + ((seed * 0x9E3779B1 + step * 0x6A09E667) & low)) & low
    x = ((x ^ (x >> 16)) * 0xBB67AE85) & low
    x = ((x ^ (x >> 15)) * 0x3C6EF373) & low
    return x ^ (x >> 16)


def _stored(x, up, bits16):
    """x in blocks of 256 as codes and scales: largest / 448 is the scale, and a value goes to the code below or above it as the 16
    random bits say, so that on average it keeps its value; up: above zero it stays above zero."""
    n = x.numel()
    blocks = torch.cat([x.reshape(-1), x.new_zeros(-n % 256)]).view(-1, 256)
    largest = blocks.abs().amax(1, keepdim=True)
    there = largest >= 2.0 ** -100
    y = torch.where(there, blocks * (448.0 / largest), torch.zeros_like(blocks)).clamp(-448.0, 448.0).view(-1)[:n].double()
    a = y.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    q = torch.floor(a / step + bits16.double() / 65536.0) * step
    if up:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    return torch.where(y < 0, -q, q).float().to(_E4M3), torch.where(there, largest * (1.0 / 448.0), torch.zeros_like(largest)).view(-1)


def _adamw_tensor(s, i):
    """Weights, moments and scales of tensor i after the step."""
    case, of, real = s["case"], s["lists"], torch.float32
    w, g = of["w"][i], of["g"][i].to(real)
    c1, c2 = 1.0 - _BETA1 ** _STEP, 1.0 - _BETA2 ** _STEP
    n, scales = w.numel(), None
    if case["bits"] == 8:
        each = lambda row: of["scales"][i][row].repeat_interleave(256)[:n].view(w.shape)  # noqa: E731
        m, v = of["m"][i].to(real) * each(0), (of["v"][i].to(real) * each(1)).square()
    else:
        m, v = of["m"][i], of["v"][i]
    m = _BETA1 * m + (1.0 - _BETA1) * g
    v = _BETA2 * v + (1.0 - _BETA2) * g * g
    r = torch.sqrt(v)
    w = w - _LR * s["decay"][i] * w
    w = w - _LR * (m / c1) / (r / math.sqrt(c2) + _ADAM_EPS)
    if of["keep"][i] is not None:
        w = w * of["keep"][i].repeat_interleave(s["rows"][i], 0).to(real)
    if case["bits"] == 8:
        bits = _bits(torch.arange(n, device=w.device), _STEP, _SEED)
        m, sm = _stored(m, False, bits & 0xFFFF)
        v, sv = _stored(r, True, bits >> 16)
        m, v, scales = m.view(w.shape), v.view(w.shape), torch.stack([sm, sv])
    return w, m, v, scales


def _adamw(s):
    of = s["lists"]
    for i in range(len(of["w"])):
        w, m, v, scales = _adamw_tensor(s, i)
        of["w"][i].copy_(w)
        of["m"][i].copy_(m)
        of["v"][i].copy_(v)
        of["copy"][i].copy_(w)
        if scales is not None:
            of["scales"][i].copy_(scales)
    return {k: s[k] for k in ("w", "m", "v", "copy", "scales") if k in s}


# ---- one pass -----------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2009_08065_amd as bsp
    case, path = s["case"], s["case"]["path"]
    if path == "layer8":
        w = bsp.Fp8(*s["w"], case["M"], case["N"], bsp.FP8_BLOCK)
        return bsp.bsp_linear_fp8(s["x"], w, s["bias"], act=bsp.ACT_GELU if case["gelu"] else bsp.ACT_NONE, residual=s["residual"])
    if path == "train8":
        x, xt = bsp.bsp_fp8_quant(s["x"], bsp.FP8_ROW, want=("plain", "transposed"))
        w, wt = bsp.bsp_fp8_quant(s["w"], bsp.FP8_BLOCK, want=("plain", "transposed"))
        dy, dyt = bsp.bsp_fp8_quant(s["dy"], bsp.FP8_ROW, want=("plain", "transposed"))
        dt = s["x"].dtype
        return {"y": bsp.bsp_matmul_fp8(x, w, out_dtype=dt), "dx": bsp.bsp_matmul_fp8(dy, wt, out_dtype=dt),
                "dw": bsp.bsp_matmul_fp8(dyt, xt, out_dtype=torch.float32)}
    if path == "adamw":
        of = s["lists"]
        bsp.bsp_adamw_step(of["w"], of["g"], of["m"], of["v"], _LR, beta1=_BETA1, beta2=_BETA2, eps=_ADAM_EPS, weight_decay=s["decay"],
                           t=_STEP, scales=of["scales"] or None, keep=of["keep"], R=s["rows"], copies=of["copy"], seed=_SEED)
        return {k: s[k] for k in ("w", "m", "v", "copy", "scales") if k in s}
    kind = bsp.NORM_LAYER if case["kind"] == _LAYER else bsp.NORM_RMS
    norms = (bsp.NORM_POST if case["post"] else 0) | (bsp.NORM_PRE if case["pre"] else 0)
    if path == "join":
        z, h, stats_post, stats_pre = bsp.bsp_block_norm(
            s["x"], s["f"], norms, kind=kind, eps=_EPS, x_scale=case["x_scale"], gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"],
            w_pre=s["w_pre"], b_pre=s["b_pre"])
        out = {"z": z, "h": h, "stats_post": stats_post, "stats_pre": stats_pre}
    else:
        out = bsp.bsp_block_norm_backward(
            s["dz"], s["dh"], s["z"], s["f"], norms, kind=kind, x_scale=case["x_scale"], gate=s["gate"], w_post=s["w_post"],
            b_post=s["b_post"], w_pre=s["w_pre"], b_pre=s["b_pre"], stats_post=s["stats_post"], stats_pre=s["stats_pre"])
    return {k: v for k, v in out.items() if v is not None}


def run(s):
    if own:
        return _own(s)
    path = s["case"]["path"]
    if path == "layer8":
        return _layer8(s)
    if path == "train8":
        return _train8(s)
    if path == "join":
        return _join(s)
    if path == "adamw":
        return _adamw(s)
    return _join_back(s)


def work(case):
    path = case["path"]
    if path == "adamw":
        n = sum(M * N for M, N, _ in _tensors(case))
        matrices = sum(M * N / _rows(case, M) for M, N, _ in _tensors(case) if M > 1)
        moments = 16.0 if case["bits"] == 32 else 4.0 + 4.0 * 4 / 256
        return {"bytes": n * (8.0 + (2.0 if case["grad"] == "bf16" else 4.0) + moments + 2.0) + (matrices if case["masked"] else 0), "flops": 15.0 * n}
    size, T = 4.0 if case["dtype"] == "f32" else 2.0, case["T"]
    if path == "layer8":
        M, N = case["M"], case["N"]
        return {"bytes": size * (T * N + T * M * (2 if case["residual"] else 1)) + M * N, "flops": 2.0 * T * M * N}
    if path == "train8":
        M, N = case["M"], case["N"]
        return {"bytes": size * (2 * T * N + 2 * T * M + M * N) + 4.0 * M * N, "flops": 6.0 * T * M * N}
    H, pre, post = case["H"], int(case["pre"]), int(case["post"])
    if path == "join":
        return {"bytes": size * T * H * (3 + pre) + 8.0 * T * (pre + post), "flops": T * H * (3.0 + 6.0 * (pre + post))}
    reads = 1 + 2 * pre + (1 if post or case["gate"] else 0)
    return {"bytes": size * T * H * (reads + 2), "flops": T * H * (3.0 + 12.0 * (pre + post))}


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------------------
def _value8(x, rows):
    """x [r, c] in 64 bits as 8-bit floating point holds it, a power of two for `rows` x 128 elements: the significand is rounded to
    four bits by hand."""
    r, c = x.shape
    p = torch.zeros((r + -r % rows, c + -c % 128), dtype=torch.float64, device=x.device)
    p[:r, :c] = x
    t = p.view(p.shape[0] // rows, rows, p.shape[1] // 128, 128)
    top = t.abs().amax(dim=(1, 3), keepdim=True)
    least = 448.0 * torch.pow(torch.tensor(2.0, dtype=torch.float64), torch.arange(-127, 122)).to(x.device)
    unit = (least / 448.0)[torch.searchsorted(least, top)]  # of the first power of two whose 448 fold is not below the largest value
    unit = torch.where(top > 0, unit, torch.ones_like(unit))
    y = t / unit
    lsb = torch.full_like(y, 2.0 ** -9)
    for k in range(-5, 9):
        lsb = torch.where(y.abs() >= 2.0 ** k, 2.0 ** (k - 3), lsb)
    return (torch.round(y / lsb) * lsb * unit).view(p.shape)[:r, :c]


def exact(case, seed):
    s = prepare(case, seed)
    path, d = case["path"], torch.float64
    if path == "layer8":
        codes, e = s["w"]
        scale = ((e.long() + 896) << 52).view(d).repeat_interleave(128, 0)[:case["M"]].repeat_interleave(128, 1)
        w = (codes.to(d) * scale)[:, :case["N"]].contiguous()
        y = torch.mm(_value8(s["x"].to(d), 1), w.t())
        if s["bias"] is not None:
            y += s["bias"].to(d)
        if case["gelu"]:
            y = 0.5 * y * torch.special.erfc(y * -math.sqrt(0.5))
        return y if s["residual"] is None else y + s["residual"].to(d)
    if path == "train8":
        x, dy, w = s["x"].to(d), s["dy"].to(d), _value8(s["w"].to(d), 128)
        return {"y": torch.mm(_value8(x, 1), w.t()), "dx": torch.mm(_value8(dy, 1), w),
                "dw": torch.mm(_value8(dy.t().contiguous(), 1), _value8(x.t().contiguous(), 1).t())}
    if path == "adamw":
        out, of = {k: [] for k in ("w", "m", "v", "copy", "scales")}, s["lists"]
        for i, decay in enumerate(s["decay"]):
            g, w, m, v = (of[k][i].reshape(-1).to(d) for k in ("g", "w", "m", "v"))
            n = g.numel()
            if case["bits"] == 8:
                block = torch.arange(n, device="cuda") // 256
                m, v = m * of["scales"][i][0].to(d)[block], (v * of["scales"][i][1].to(d)[block]) ** 2
            m, v = m + (g - m) * (1 - _BETA1), v + (g ** 2 - v) * (1 - _BETA2)
            w = w * (1 - _LR * decay) - _LR * m / (1 - _BETA1 ** _STEP) / ((v / (1 - _BETA2 ** _STEP)) ** 0.5 + _ADAM_EPS)
            if of["keep"][i] is not None:
                M, N = of["w"][i].shape
                w = (w.view(-1, s["rows"][i], N) * of["keep"][i].to(d)[:, None, :]).view(-1)
            if case["bits"] == 8:
                word = _bits(torch.arange(n, device="cuda"), _STEP, _SEED)
                held = []
                for x, u in ((m, word % 65536), (v ** 0.5, word // 65536)):
                    top = torch.zeros(int(block[-1]) + 1, dtype=d, device="cuda").scatter_reduce_(0, block, x.abs(), "amax")
                    y = x * (448 / top)[block]
                    k = torch.frexp(y.abs()).exponent.clamp(min=-5)  # |y| < 2^k
                    unit = torch.pow(2.0, (k - 4).to(d))
                    q = torch.trunc(y.abs() / unit + u.to(d) / 65536) * unit
                    if x is not m:
                        q = torch.where((q == 0) & (y > 0), 2.0 ** -9, q)
                    held.append((q.clamp(max=448) * torch.sign(y), top / 448))
                (m, sm), (v, sv) = held
                out["scales"] += [sm, sv]
            for k, t in (("w", w), ("m", m), ("v", v), ("copy", w)):
                out[k].append(t)
        return {k: torch.cat(v) for k, v in out.items() if v}
    T, H = case["T"], case["H"]
    f = s["f"].to(d)
    if path == "join":
        def moments(x):
            mu = x.sum(1) / H if case["kind"] == _LAYER else torch.zeros(T, dtype=d, device="cuda")
            return mu, torch.rsqrt(((x - mu[:, None]) ** 2).sum(1) / H + _EPS)
        out = {}
        if case["post"]:
            mu, rs = moments(f)
            out["stats_post"] = torch.stack([mu, rs], 1)
            f = (f - mu[:, None]) * rs[:, None] * s["w_post"].to(d)
            if s["b_post"] is not None:
                f = f + s["b_post"].to(d)
        if case["gate"]:
            f = (f.view(case["gate"], -1, H) * s["gate"].to(d)[:, None, :]).view(T, H)
        out["z"] = s["x"].to(d) * case["x_scale"] + f
        if case["pre"]:
            z = out["z"].to(s["x"].dtype).to(d)
            mu, rs = moments(z)
            out["stats_pre"] = torch.stack([mu, rs], 1)
            out["h"] = (z - mu[:, None]) * rs[:, None] * s["w_pre"].to(d) + (0.0 if s["b_pre"] is None else s["b_pre"].to(d))
        return out
    # the gradients by automatic differentiation of the norms, their statistics taken as they were kept
    leaf = lambda t: None if t is None else t.to(d).requires_grad_()  # noqa: E731
    x, f, gate, wp, bp, wq, bq = (leaf(t) for t in (s["z"] if case["pre"] else s["x"], s["f"], s["gate"], s["w_post"], s["b_post"], s["w_pre"], s["b_pre"]))

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, v, stats):
            hat = (v - stats[:, :1]) * stats[:, 1:]
            ctx.save_for_backward(hat, stats)
            return hat

        @staticmethod
        def backward(ctx, dy):
            hat, stats = ctx.saved_tensors
            back = dy - hat * (dy * hat).sum(1, keepdim=True) / H
            return (back - (dy.sum(1, keepdim=True) / H if case["kind"] == _LAYER else 0.0)) * stats[:, 1:], None
    out, dz = {}, s["dz"].to(d)
    with torch.enable_grad():
        if case["pre"]:
            h = Norm.apply(x, s["stats_pre"].to(d)) * wq
            h = h if bq is None else h + bq
            grads = torch.autograd.grad(h, [t for t in (x, wq, bq) if t is not None], s["dh"].to(d))
            dz, out["dw_pre"], out["db_pre"] = dz + grads[0], grads[1], grads[2] if bq is not None else None
        n = f * 1.0
        if case["post"]:
            n = Norm.apply(f, s["stats_post"].to(d)) * wp
            n = n if bp is None else n + bp
        if case["gate"]:
            n = (n.view(case["gate"], -1, H) * gate[:, None, :]).view(T, H)
        names = [k for k, t in (("df", f), ("dgate", gate), ("dw_post", wp), ("db_post", bp)) if t is not None]
        out.update(zip(names, torch.autograd.grad(n, [t for t in (f, gate, wp, bp) if t is not None], dz)))
    out["dx"] = dz * case["x_scale"]
    return {k: v for k, v in out.items() if v is not None}
