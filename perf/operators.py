"""The feed-forward training step's operators beside the integer layers, on the sizes they are measured on:
layer norm (forward, backward), 8-bit floating point layers with a scale for each block of 128 (forward,
backward, the weights' quantizer) and the global gradient norm with clipping.

A case is a dict of plain values:

  op      "norm_forward", "norm_backward", "fp8_forward", "fp8_backward", "fp8_weights" or "clip"
  dtype   "f32", "bf16" or "f16": activations and their gradients (clip: the gradients); weights and
          parameter gradients are float32

``run`` is one pass: in elementary torch operations where ``own`` is false, through the library where it is
true.  ``exact`` is the same from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
FP8_MAX = 448.0  # largest value of the 8-bit format with 4 exponent and 3 mantissa bits


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _norm(name, way, rows, cols, dtype):
    return dict(name=name, op="norm_" + way, rows=rows, cols=cols, dtype=dtype)


def _fp8(name, way, N, d_in, d_out, dtype, relu=False, save=True):
    case = dict(name=name, op="fp8_" + way, N=N, d_in=d_in, d_out=d_out, dtype=dtype, relu=relu)
    return dict(case, save=save) if way == "forward" else case


def _resnet50_sizes():
    """Weights of ResNet-50's 53 convs with their norms' two vectors, and the classifier."""
    convs, c = [64 * 3 * 49], 64
    norms = [64]
    for width, out, blocks in ((64, 256, 3), (128, 512, 4), (256, 1024, 6), (512, 2048, 3)):
        for b in range(blocks):
            convs += [c * width, 9 * width * width, width * out] + ([c * out] if b == 0 else [])
            norms += [width, width, out] + ([out] if b == 0 else [])
            c = out
    sizes = [n for w, d in zip(convs, norms) for n in (w, d, d)]
    return ",".join(str(n) for n in sizes + [2048 * 1000, 1000])


def listed():
    return [
        # one token's activations in front of a layer while serving
        _norm("norm_forward_token", "forward", 1, 4096, "bf16"),
        # the feed-forward layer's hidden width over a whole training batch
        _norm("norm_forward_batch", "forward", 8192, 4096, "f32"),
        # the benchmark layer's input width, the batch of a training step in half-length activations
        _norm("norm_backward_batch", "backward", 8192, 1024, "bf16"),
        # a ragged batch of an odd width
        _norm("norm_backward_odd", "backward", 3001, 1001, "f16"),
        # serving: one token through the benchmark's layer, whose codes the server keeps
        _fp8("fp8_forward_token", "forward", 1, 1024, 4096, "bf16", save=False),
        # the classifier layer of the measured workloads: rows, columns and outputs off every tile
        _fp8("fp8_forward_odd", "forward", 250, 2048, 1001, "f32"),
        # the benchmark's feed-forward up-projection with its ReLU, keeping what grad_W reads
        _fp8("fp8_forward_ffn", "forward", 8192, 1024, 4096, "bf16", relu=True),
        # that layer's backward: stochastic codes of the gradient, both products
        _fp8("fp8_backward_ffn", "backward", 8192, 1024, 4096, "bf16"),
        # the down-projection's backward on a ragged batch, behind a ReLU
        _fp8("fp8_backward_ragged", "backward", 3001, 4096, 1024, "f32", relu=True),
        # once a step: the float32 weights into codes for the forward and for grad_X
        _fp8("fp8_weights", "weights", 0, 1024, 4096, "f32"),
        # the gradients of the benchmark's three-layer chain 1024-4096-4096-1024
        dict(name="clip_chain", op="clip", sizes="4194304,16777216,4194304", dtype="f32", max_norm=1.0),
        # a network of many small tensors in one bucket: ResNet-50's 161
        dict(name="clip_many", op="clip", sizes=_resnet50_sizes(), dtype="bf16", max_norm=1.0),
    ]


MAX_FLOPS = 1.38e11
MAX_BYTES = 2.7e8


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, step=16):
    """Log-uniform; half of the draws rounded up to a multiple of step, half as they fall."""
    v = _log_int(rng, lo, hi)
    return (v + step - 1) // step * step if rng.random() < 0.5 else v


def draw(rng):
    """One more case of the listed ones' ranges: 1 .. 8192 tokens, widths 64 .. 4096, 1 .. 200 gradient tensors
    of 1 .. 16 M elements, every type."""
    while True:
        op = rng.choice(["norm_forward", "norm_backward", "fp8_forward", "fp8_forward", "fp8_backward",
                         "fp8_backward", "fp8_weights", "clip"])
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        if op.startswith("norm"):
            case = dict(op=op, rows=_size(rng, 1, 8192), cols=_size(rng, 64, 4096), dtype=dtype)
        elif op == "clip":
            sizes = [_log_int(rng, 1, 1 << 24) for _ in range(_log_int(rng, 1, 200))]
            case = dict(op=op, sizes=",".join(map(str, sizes)), dtype=dtype, max_norm=rng.choice([0.1, 1.0, 1e6]))
        else:
            case = dict(op=op, N=_size(rng, 1, 8192), d_in=_size(rng, 64, 4096), d_out=_size(rng, 64, 4096),
                        dtype=dtype, relu=rng.random() < 0.5)
            if op == "fp8_forward":
                case["save"] = rng.random() < 0.5
            if op == "fp8_weights":
                case.update(N=0, relu=False, dtype="f32")
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return case


def work(case):
    """Bytes: each input read once, each output written once (codes one byte).  Flops: the products, and about
    eight operations an element in a norm, two in a clip."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("norm"):
        n, back = case["rows"] * case["cols"], case["op"] == "norm_backward"
        return {"bytes": (3.0 if back else 2.0) * e * n + 12.0 * case["cols"] + 8.0 * case["rows"], "flops": 8.0 * n}
    if case["op"] == "clip":
        n = sum(map(int, case["sizes"].split(",")))
        return {"bytes": 2.0 * e * n, "flops": 4.0 * n}
    N, i, o = case["N"], case["d_in"], case["d_out"]
    if case["op"] == "fp8_weights":
        return {"bytes": 6.0 * i * o, "flops": 2.0 * i * o}
    if case["op"] == "fp8_forward":
        return {"bytes": 1.0 * e * N * (i + o) + i * o + (N * i if case["save"] else 0), "flops": 2.0 * N * i * o}
    mask = e * N * i if case["relu"] else 0
    return {"bytes": 1.0 * e * N * (i + o) + N * i + 5.0 * i * o + mask, "flops": 4.0 * N * i * o}


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _gradient(normal, gen, rows, cols):
    """An output gradient: 1 % large rows (0.5 % of none: masked tokens), the rest small."""
    kind = torch.rand((rows, 1), generator=gen, device=DEV)
    return normal((rows, cols)).mul_(torch.where(kind < 0.01, 10.0, torch.where(kind > 0.995, 0.0, 0.01)))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(shape, std=1.0):
        return torch.randn(shape, generator=gen, device=DEV).mul_(std)

    st = dict(case=dict(case), seed=int(seed) % (1 << 31))
    if case["op"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        # a residual stream: rows of unlike size with a mean of their own, a few large channels
        x = normal((rows, cols)).mul_(torch.exp(0.5 * normal((rows, 1)))).add_(normal((rows, 1), 0.5))
        x *= torch.where(torch.rand(cols, generator=gen, device=DEV) < 0.01, 8.0, 1.0)
        st["x"] = x.to(dt)
        st["gamma"], st["beta"] = 1.0 + normal(cols, 0.1), normal(cols, 0.1)
        if case["op"] == "norm_backward":
            st["g"] = _gradient(normal, gen, rows, cols).to(dt)
            mean, rstd = _row_statistics(st["x"].double())
            st["mean"], st["rstd"] = mean.float().view(-1), rstd.float().view(-1)
    elif case["op"] == "clip":
        sizes = [int(n) for n in case["sizes"].split(",")]
        scale = torch.exp(normal(len(sizes)) - 5.0)
        flat = normal(sum(sizes)).mul_(torch.repeat_interleave(scale, torch.tensor(sizes, device=DEV)))
        st["flat"] = flat.to(dt)  # one bucket, a tensor behind the other
        st["out_flat"] = torch.empty_like(st["flat"])
        st["grads"], st["outs"] = list(st["flat"].split(sizes)), list(st["out_flat"].split(sizes))
    else:
        N, i, o = case["N"], case["d_in"], case["d_out"]
        W = normal((o, i), i ** -0.5)
        if case["op"] == "fp8_weights":
            st["W"] = W
            return st
        X = normal((N, i)).to(dt)
        if case["op"] == "fp8_forward":
            st["X"], st["W8"] = X, _operand(W, tile=True)
        else:
            st["X"] = X.clamp_(min=0.0) if case["relu"] else None
            st["G"] = _gradient(normal, gen, N, o).to(dt)
            # what the forward kept: the activations and weights as the backward's products read them
            st["X8t"], st["W8t"] = _operand(X.float().t()), _operand(W.t(), tile=True)
    return st


# ----------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------
def _row_statistics(x):
    mean = x.mean(1, keepdim=True)
    return mean, 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)


def _words(rows, cols, seed, stream):
    """The 24-bit uniform of every element: Philox4x32-7, counter = element index / 4, as float32."""
    total, mask = rows * cols, 0xFFFFFFFF
    blk = torch.arange((total + 3) // 4, dtype=torch.int64, device=DEV)
    c0, c1, c2, c3 = blk & mask, blk >> 32, torch.full_like(blk, stream), torch.zeros_like(blk)
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(7):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # products modulo 2^64
        c0, c1, c2, c3 = (((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask)
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    u = torch.stack([w.bitwise_and(0xFFFFFF).float() for w in (c0, c1, c2, c3)], dim=1)
    return u.view(-1)[:total].view(rows, cols)


def _operand(x, tile=False, u=None):
    """The codes of x [rows, K] in blocks of 128 along K, each with the least power of two 2^E that brings it
    within the format (tile: one for 128 x 128), nearest-even or, with uniforms u, stochastic:
    {"q": codes [rows, K padded to whole blocks], "exp": E + 127 of block b at [b / 4, row, b % 4], "K"}."""
    rows, K = x.shape
    kb = -(-K // 128)
    x = torch.nn.functional.pad(x.float(), (0, kb * 128 - K)).view(rows, kb, 128)
    top = x.abs().amax(2)
    if tile:
        rb = -(-rows // 128)
        top = torch.nn.functional.pad(top, (0, 0, 0, rb * 128 - rows)).view(rb, 128, kb).amax(1)
        top = top.repeat_interleave(128, 0)[:rows]
    m, p = torch.frexp(top)
    e = torch.where(top > 0, (p - 9 + (m > 0.875).int()).clamp(min=-127), 0)
    y = torch.ldexp(x, -e[:, :, None])
    if u is not None:
        u = torch.nn.functional.pad(u, (0, kb * 128 - K)).view(rows, kb, 128)
        step = (torch.frexp(y.abs())[1] - 1).clamp(min=-6) - 3  # spacing of the format's values around y
        t = torch.ldexp(y.abs(), -step)
        fl = t.floor()
        y = torch.copysign(torch.ldexp(fl + (u < (t - fl) * 16777216.0), step), y)
    exp = torch.full((rows, -(-kb // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    exp[:, :kb] = (e + 127).to(torch.uint8)
    return {"q": y.view(rows, kb * 128).to(torch.float8_e4m3fn), "K": K,
            "exp": exp.view(rows, -1, 4).transpose(0, 1).contiguous()}


def _values(a):
    """The float32 values that an operand stands for."""
    rows, ld = a["q"].shape
    e = a["exp"].transpose(0, 1).reshape(rows, -1)[:, :ld // 128].to(torch.int32) - 127
    return torch.ldexp(a["q"].float().view(rows, -1, 128), e[:, :, None]).view(rows, ld)


def _codes(a):
    return {"q": a["q"], "exp": a["exp"]}


def _run_plain(st):
    case = st["case"]
    dt = TYPES[case["dtype"]]
    if case["op"] == "norm_forward":
        x = st["x"].float()
        mean, rstd = _row_statistics(x)
        y = (x - mean) * rstd * st["gamma"] + st["beta"]
        return {"Y": y.to(dt), "mean": mean.view(-1), "rstd": rstd.view(-1)}
    if case["op"] == "norm_backward":
        g, rstd = st["g"].float(), st["rstd"].view(-1, 1)
        xh = (st["x"].float() - st["mean"].view(-1, 1)) * rstd
        c = g * st["gamma"]
        gx = rstd * (c - c.mean(1, keepdim=True) - xh * (c * xh).mean(1, keepdim=True))
        return {"grad_X": gx.to(dt), "grad_gamma": (g * xh).sum(0), "grad_beta": g.sum(0)}
    if case["op"] == "clip":
        norm = torch.sqrt(torch.stack([g.float().square().sum() for g in st["grads"]]).sum())
        scale = torch.where(norm > case["max_norm"], case["max_norm"] / norm, 1.0)
        [o.copy_(g.float() * scale) for g, o in zip(st["grads"], st["outs"])]
        return {"norm": norm, "grads": st["out_flat"]}
    if case["op"] == "fp8_weights":
        return {"W8": _codes(_operand(st["W"], tile=True)), "W8t": _codes(_operand(st["W"].t(), tile=True))}
    if case["op"] == "fp8_forward":
        Y = _values(_operand(st["X"])) @ _values(st["W8"]).t()
        out = {"Y": (Y.clamp(min=0.0) if case["relu"] else Y).to(dt)}
        return dict(out, X8t=_codes(_operand(st["X"].t()))) if case["save"] else out
    G = st["G"]
    rows, cols = G.shape
    G1 = _values(_operand(G.t(), u=_words(rows, cols, st["seed"], 0).t()))
    G2 = _values(_operand(G, u=_words(rows, cols, st["seed"], 1)))
    gX = G2 @ _values(st["W8t"]).t()
    if case["relu"]:
        gX = gX * (st["X"] > 0)
    return {"grad_W": G1 @ _values(st["X8t"]).t(), "grad_X": gX.to(dt)}


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(st):
    if not own:
        return _run_plain(st)
    from paper_2010_14298_amd import fqt
    case = st["case"]
    if case["op"] == "norm_forward":
        Y, mean, rstd = fqt.fqt_layernorm_forward(st["x"], st["gamma"], st["beta"], eps=EPS)
        return {"Y": Y, "mean": mean, "rstd": rstd}
    if case["op"] == "norm_backward":
        gX, gg, gb, _ = fqt.fqt_layernorm_backward(st["g"], st["x"], st["mean"], st["rstd"], st["gamma"])
        return {"grad_X": gX, "grad_gamma": gg, "grad_beta": gb}
    if case["op"] == "clip":
        norm, _ = fqt.fqt_grad_norm_clip(st["grads"], case["max_norm"], outs=st["outs"])
        return {"norm": norm, "grads": st["out_flat"]}
    if case["op"] == "fp8_weights":
        W8, W8t = fqt.fqt_fp8_quantize(st["W"], tile=True, by_row=True, by_col=True)
        return {"W8": _codes(W8), "W8t": _codes(W8t)}
    if case["op"] == "fp8_forward":
        Y, X8t, _ = fqt.fqt_fp8_linear_forward(st["X"], st["W8"], relu=case["relu"], save=case["save"])
        return {"Y": Y, "X8t": _codes(X8t)} if case["save"] else {"Y": Y}
    gW, gX, _ = fqt.fqt_fp8_linear_backward(st["G"], st["X8t"], st["W8t"], seed=st["seed"], relu_input=st["X"])
    return {"grad_W": gW, "grad_X": gX}


# ----------------------------------------------------------------------------
# the reference
# ----------------------------------------------------------------------------
def _exact_uniforms(rows, cols, seed, stream):
    """The same stream in 64-bit unsigned numpy arithmetic: float64 in [0, 2^24)."""
    n, m32, s32 = (rows * cols + 3) // 4, np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.arange(n, dtype=np.uint64) & m32, np.arange(n, dtype=np.uint64) >> s32,
         np.full(n, stream, dtype=np.uint64), np.zeros(n, dtype=np.uint64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        ka, kb = ((key[j] + r * w) & 0xFFFFFFFF for j, w in ((0, 0x9E3779B9), (1, 0xBB67AE85)))
        c = [(b >> s32) ^ c[1] ^ np.uint64(ka), b & m32, (a >> s32) ^ c[3] ^ np.uint64(kb), a & m32]
    w = np.stack([v & np.uint64(0xFFFFFF) for v in c], axis=1).reshape(-1)[:rows * cols]
    return torch.from_numpy(w.astype(np.float64)).to(DEV).view(rows, cols)


def _exact_blocks(x, tile, u=None):
    """(codes, values, exponents + 127) of float64 x [rows, K]: the block exponent by comparing the largest
    magnitude with 448 times each power of two near it, the code by counting steps of the format at y."""
    rows, K = x.shape
    h, kb = (128 if tile else 1), -(-K // 128)
    rb = -(-rows // h)
    big = torch.zeros((rb * h, kb * 128), dtype=torch.float64, device=DEV)
    big[:rows, :K] = x
    top = big.view(rb, h, kb, 128).abs().amax((1, 3))
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0) / FP8_MAX)) - 1
    for _ in range(3):
        e += (top > FP8_MAX * torch.exp2(e)).double()
    e = torch.where(top > 0, e.clamp(min=-127), 0.0)
    scale = torch.exp2(e)[:, None, :, None].expand(rb, h, kb, 128).reshape(rb * h, kb * 128)[:rows]
    y = (big[:rows] / scale).abs()
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    t = y / step
    if u is None:
        n = torch.round(t)
    else:
        wide = torch.zeros((rows, kb * 128), dtype=torch.float64, device=DEV)
        wide[:, :K] = u
        n = torch.floor(t) + (wide < (t - torch.floor(t)) * 2.0 ** 24)
    q = torch.sign(big[:rows]) * n * step
    exp = torch.full((-(-kb // 4) * 4, rows), 127, dtype=torch.uint8, device=DEV)
    exp[:kb] = (e.t().repeat_interleave(h, 1)[:, :rows] + 127).to(torch.uint8)
    return q, q * scale, exp.view(-1, 4, rows).transpose(1, 2).contiguous()


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"].startswith("norm"):
        x, gamma, n = st["x"].double(), st["gamma"].double(), case["cols"]
        mean = x.sum(1, keepdim=True) / n
        d = x - mean
        r = ((d * d).sum(1, keepdim=True) / n + EPS) ** -0.5
        if case["op"] == "norm_forward":
            return {"Y": d * r * gamma + st["beta"].double(), "mean": mean.view(-1), "rstd": r.view(-1)}
        g = st["g"].double()
        a, b = (g * gamma).sum(1, keepdim=True) / n, (g * gamma * d).sum(1, keepdim=True) / n
        return {"grad_X": r * (g * gamma - a) - d * b * r ** 3, "grad_gamma": (g * d * r).sum(0),
                "grad_beta": g.sum(0)}
    if case["op"] == "clip":
        g = st["flat"].double()
        norm = torch.linalg.vector_norm(g)
        return {"norm": norm, "grads": g * min(1.0, case["max_norm"] / float(norm))}
    if case["op"] == "fp8_weights":
        W = st["W"].double()
        (a, _, ae), (b, _, be) = _exact_blocks(W, True), _exact_blocks(W.t(), True)
        return {"W8": {"q": a, "exp": ae}, "W8t": {"q": b, "exp": be}}
    if case["op"] == "fp8_forward":
        X = st["X"].double()
        Y = _exact_blocks(X, False)[1] @ _values(st["W8"]).double().t()
        out = {"Y": Y.clamp(min=0.0) if case["relu"] else Y}
        if case["save"]:
            q, _, e = _exact_blocks(X.t(), False)
            out["X8t"] = {"q": q, "exp": e}
        return out
    G = st["G"].double()
    rows, cols = G.shape
    G1 = _exact_blocks(G.t(), False, _exact_uniforms(rows, cols, st["seed"], 0).t())[1]
    G2 = _exact_blocks(G, False, _exact_uniforms(rows, cols, st["seed"], 1))[1]
    gX = G2 @ _values(st["W8t"]).double().t()
    if case["relu"]:
        gX = torch.where(st["X"] > 0, gX, 0.0)
    return {"grad_W": G1 @ _values(st["X8t"]).double().t(), "grad_X": gX}
