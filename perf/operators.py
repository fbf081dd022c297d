"""Workloads of the linear layer around the sparse product, for timing: the product with bias, activation and residual, 8-bit
activation checkpoints, the gradient through the activation, the dense weight gradient.

  linear      Z = X (B .* W)^T + bias,  Y = act(Z) + residual, and (ckpt) Z kept in 8 bits for the backward pass
  checkpoint  X into 8 bits and back: 32 consecutive features of a token share a power of two 2^e, the smallest with
              rint(max|x| / 2^e) <= 127 (-126 <= e <= 121); a feature is rint(x / 2^e) within +-127, halves to even
  act_grad    dZ = dY * act'(Z~) and dbias = sum over the tokens of dZ, Z~ being what the checkpoint of Z stands for
  weight_grad dW = dY^T X~, X~ being what the checkpoint of X stands for

A checkpoint is one byte buffer: T rows of codes (signed, the row padded with zeros to a multiple of 32), then for every row one byte
e + 127 per 32 features (255: the 32 features hold an infinity or NaN and read as NaN).  Sizes are those of this repository's
configurations (`paper_2302_06058_amd/synth.py`) and generic ones.
"""
import math

import torch

own = False


def listed():
    def linear(name, I, J, T, act, N=2, M=4, dtype="bf16", bias=True, residual=False, ckpt=False):
        return dict(name=name, op="linear", dtype=dtype, N=N, M=M, I=I, J=J, T=T, act=act, bias=bias, residual=residual, ckpt=ckpt)

    return [
        # the smallest layer of the configurations, everything on: bound by latency
        linear("linear-f32-small", 64, 128, 32, "gelu", dtype="f32", residual=True),
        # serving: the first matrix of a transformer MLP for a single token
        linear("decode-up", 11008, 4096, 1, "silu", bias=False),
        # serving: its second matrix for a few sequences at once, onto the residual stream
        linear("decode-down-batch", 4096, 11008, 13, "none", bias=False, residual=True),
        # training, small vision transformer at 128 images: first MLP matrix on dense matrix instructions, pre-activation kept
        linear("fc1-4of8-train", 1536, 384, 25216, "gelu", N=4, M=8, ckpt=True),
        # its second MLP matrix at 1:4, onto the residual stream, a token count that fills no tile
        linear("fc2-1of4-residual", 384, 1536, 25211, "none", N=1, residual=True),
        # training of a large transformer MLP: the largest product, pre-activation kept
        linear("mlp-up-train", 11008, 4096, 8192, "silu", bias=False, ckpt=True),
        # fp32 features of an odd width and few tokens
        dict(name="checkpoint-f32-odd", op="checkpoint", dtype="f32", T=197, J=1001),
        # the hidden activations of the large MLP
        dict(name="checkpoint-mlp", op="checkpoint", dtype="bf16", T=8192, J=11008),
        # the classifier's hidden layer: ragged width
        dict(name="act-grad-head", op="act_grad", dtype="bf16", T=6347, I=1000, act="gelu"),
        # the large MLP's hidden layer
        dict(name="act-grad-mlp", op="act_grad", dtype="bf16", T=8192, I=11008, act="silu"),
        # 3x3 convolution of the first stage: a long contraction onto few weights
        dict(name="weight-grad-conv", op="weight_grad", dtype="bf16", dw="f32", I=64, J=576, T=200704),
        # the large MLP's first matrix
        dict(name="weight-grad-mlp", op="weight_grad", dtype="bf16", dw="bf16", I=11008, J=4096, T=8192),
    ]


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
RATIOS = ((2, 4), (2, 4), (2, 4), (1, 4), (4, 8), (2, 8), (1, 16))


def draw(rng):
    def spread(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))

    def size(lo, hi, step):
        """Spread over the logarithm; half on multiples of 32, the others on the smallest step allowed."""
        s = step if rng.random() < 0.5 else max(32, step)
        return max(s, round(spread(lo, hi) / s) * s)

    op = rng.choice(("linear", "linear", "linear", "checkpoint", "act_grad", "weight_grad", "weight_grad"))
    f32 = rng.random() < 0.15
    if op == "linear":
        N, M = rng.choice(RATIOS)
        c = dict(op=op, dtype="f32" if f32 else "bf16", N=N, M=M, act=rng.choice(ACTS), bias=rng.random() < 0.7, residual=rng.random() < 0.4)
        if f32:
            c.update(I=size(32, 1024, M), J=size(32, 1024, M), T=round(spread(1, 1024)), ckpt=False)
        else:
            serving = rng.random() < 0.4
            c.update(I=size(64, 11008, M), J=size(64, 11008, M), ckpt=not serving and rng.random() < 0.5)
            c["J"] = max(M, min(c["J"], 11008 * 4096 // c["I"] // M * M))
            c["T"] = round(spread(1, 64) if serving else spread(65, min(32768, 8192 * 11008 * 4096 // (c["I"] * c["J"]))))
        return c
    if op == "checkpoint":
        J = round(spread(17, 11008))
        return dict(op=op, dtype="f32" if f32 else "bf16", T=round(spread(1, min(65536, 8192 * 5504 // J))), J=J)
    if op == "act_grad":
        I = round(spread(17, 11008))
        return dict(op=op, dtype="f32" if f32 else "bf16", T=round(spread(1, min(65536, 8192 * 5504 // I))), I=I, act=rng.choice(ACTS[1:]))
    if f32:
        return dict(op=op, dtype="f32", dw="f32", I=size(17, 1024, 1), J=size(17, 1024, 1), T=round(spread(1, 4096)))
    I, J = size(32, 11008, 1), size(32, 11008, 1)
    J = max(1, min(J, 11008 * 4096 // I))
    return dict(op=op, dtype="bf16", dw=rng.choice(("bf16", "f32")), I=I, J=J, T=round(spread(16, min(200704, 8192 * 11008 * 4096 // (I * J), 200704 * 640 // (I + J)))))


TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, std, dt):
    return torch.empty((rows, cols), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dt)


def _features(g, rows, cols, dt):
    """Activations as they occur: unit normal, one feature in 64 much larger than the others."""
    large = torch.rand((cols,), device="cuda", generator=g) < 1 / 64
    return (_normal(g, rows, cols, 1.0, torch.float32) * torch.where(large, 12.0, 1.0)).to(dt)


def _mask(W, N, M):
    """The N largest magnitudes of every M weights of a row, the lowest index first among equals."""
    a = W.float().abs().view(W.shape[0], -1, M)
    at = torch.arange(M, device=W.device)
    first = (a.unsqueeze(-2) > a.unsqueeze(-1)) | ((a.unsqueeze(-2) == a.unsqueeze(-1)) & (at.view(1, M) < at.view(M, 1)))
    return (first.sum(-1) < N).view(W.shape)


def _operand(W, keep, N):
    """The compressed operand (layout of include/bimask.h): 2-of-4 values and index words, or for N > 2 the dense masked matrix."""
    rows, cols = W.shape
    Rp, Cp = -(-rows // 32) * 32, -(-cols // 128) * 128
    R, S = Rp // 32, Cp // 128
    w = torch.zeros((Rp, Cp), dtype=W.dtype, device=W.device)
    w[:rows, :cols] = W * keep
    if N > 2:
        return w.view(R, 32, S, 2, 4, 2, 8).permute(0, 2, 4, 3, 5, 1, 6).contiguous().view(-1), None
    k = torch.zeros((Rp, Cp), dtype=torch.int8, device=W.device)
    k[:rows, :cols] = keep
    at = torch.arange(4, device=W.device, dtype=torch.int8)
    # the mask's ones in front, then the zeros, either by position; the two first are the slots, in ascending order
    slots = ((1 - k.view(Rp, -1, 4)) * 4 + at).topk(2, dim=-1, largest=False).values.remainder(4).sort(dim=-1).values.long()
    values = w.view(Rp, -1, 4).gather(-1, slots).view(R, 32, S, 2, 4, 8).permute(0, 2, 4, 3, 1, 5).contiguous().view(-1)
    nibble = slots[..., 0] | slots[..., 1] << 2
    nibble[rows:] = 0
    nibble[:, cols // 4:] = 0
    word = (nibble.view(R, 32, S, 2, 2, 8) << 4 * torch.arange(8, device=W.device)).sum(-1)
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
    return values, word.permute(0, 2, 3, 1, 4).contiguous().view(-1)


def _quantized(x):
    """(codes, exponents) of fp32 rows, padded to whole blocks of 32: codes (T, blocks, 32) in fp32, exponents (T, blocks) integer."""
    T, J = x.shape
    b = torch.nn.functional.pad(x, (0, -J % 32)).view(T, -1, 32)
    most = b.abs().amax(dim=-1)
    m, p = torch.frexp(most)
    e = torch.where(m < 127.5 / 128, p - 7, p - 6).clamp(-126, 121)
    return torch.round(torch.ldexp(b, -e.unsqueeze(-1))).clamp(-127, 127), e, ~torch.isfinite(most)


def _kept(x, dt):
    """What the 8-bit checkpoint of fp32 rows stands for."""
    q, e, bad = _quantized(x)
    v = torch.where(bad.unsqueeze(-1), math.nan, torch.ldexp(q, e.unsqueeze(-1)))
    return v.view(x.shape[0], -1)[:, :x.shape[1]].to(dt)


def _checkpoint(x):
    """The checkpoint's byte buffer: codes, then exponents."""
    q, e, bad = _quantized(x.float())
    codes = torch.where(bad.unsqueeze(-1), 0.0, q).to(torch.int8).view(torch.uint8)
    return torch.cat((codes.reshape(-1), torch.where(bad, 255, e + 127).to(torch.uint8).reshape(-1)))


def _restored(ckpt, T, cols):
    """The values of a checkpoint's byte buffer, fp32."""
    Cp = -(-cols // 32) * 32
    codes = ckpt[:T * Cp].view(torch.int8).view(T, -1, 32).float()
    s = ckpt[T * Cp:T * Cp + T * Cp // 32].view(T, -1, 1).int()
    return torch.where(s == 255, math.nan, torch.ldexp(codes, s - 127)).view(T, Cp)[:, :cols]


def prepare(case, seed):
    g, dt, op = _generator(seed), TYPES[case["dtype"]], case["op"]
    state = dict(case=dict(case), dt=dt)
    if op == "linear":
        I, J, T, N, M = (case[k] for k in "IJTNM")
        W = _normal(g, I, J, 1.0 / math.sqrt(J * N / M), dt)
        keep = _mask(W, N, M)
        state["values"], state["index"] = _operand(W, keep, N)
        state["W"] = W * keep
        state["X"] = _features(g, T, J, dt)
        state["bias"] = _normal(g, 1, I, 0.5, dt).view(I) if case["bias"] else None
        state["residual"] = _normal(g, T, I, 1.0, dt) if case["residual"] else None
    elif op == "checkpoint":
        state["X"] = _features(g, case["T"], case["J"], dt)
    elif op == "act_grad":
        state["dY"] = _normal(g, case["T"], case["I"], 1e-2, dt)
        state["ckpt"] = _checkpoint(_normal(g, case["T"], case["I"], 1.5, dt))
    else:
        state["dY"] = _normal(g, case["T"], case["I"], 1e-2, dt)
        state["ckpt"] = _checkpoint(_features(g, case["T"], case["J"], dt))
    return state


def _act(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, 1.0)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(c * (z + 0.044715 * z * z * z))
        return s + z * s * (1.0 - s) * c * (1.0 + 3.0 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1.0 + z * (1.0 - s))


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2302_06058_amd as bm
    c = state["case"]
    if c["op"] == "linear":
        Y, ckpt = bm.bimask_sparse_linear_fwd(state["X"], state["values"], state["index"], c["I"], c["J"], c["N"], c["M"], bias=state["bias"],
                                              act=bm.ACTS[c["act"]], residual=state["residual"], want_ckpt=c["ckpt"])
        return {"Y": Y, "Z": bm.bimask_checkpoint_load(ckpt, c["T"], c["I"], state["dt"])} if c["ckpt"] else {"Y": Y}
    if c["op"] == "checkpoint":
        return {"X": bm.bimask_checkpoint_load(bm.bimask_checkpoint_store(state["X"]), c["T"], c["J"], state["dt"])}
    if c["op"] == "act_grad":
        dZ, dbias = bm.bimask_act_bwd(state["dY"], state["ckpt"], bm.ACTS[c["act"]])
        return {"dZ": dZ, "dbias": dbias}
    return {"dW": bm.bimask_weight_grad(state["dY"], state["ckpt"], c["J"], dw_dtype=TYPES[c["dw"]])}


def _run_plain(state):
    c, dt = state["case"], state["dt"]
    if c["op"] == "linear":
        Z = state["X"].float() @ state["W"].float().t()
        if state["bias"] is not None:
            Z = Z + state["bias"].float()
        Y = _act(Z, c["act"])
        if state["residual"] is not None:
            Y = Y + state["residual"].float()
        return {"Y": Y.to(dt), "Z": _kept(Z, dt)} if c["ckpt"] else {"Y": Y.to(dt)}
    if c["op"] == "checkpoint":
        return {"X": _kept(state["X"].float(), dt)}
    if c["op"] == "act_grad":
        dZ = state["dY"].float() * _act_slope(_restored(state["ckpt"], c["T"], c["I"]), c["act"])
        return {"dZ": dZ.to(dt), "dbias": dZ.sum(dim=0, dtype=torch.float64).float()}
    return {"dW": (state["dY"].float().t() @ _restored(state["ckpt"], c["T"], c["J"])).to(TYPES[c["dw"]])}


def work(case):
    """Inputs read once, outputs written once; multiplications by kept weights only (N of M)."""
    esz, T = 4 if case["dtype"] == "f32" else 2, case["T"]

    def ckpt(cols):
        return T * -(-cols // 32) * 33

    if case["op"] == "linear":
        I, J = case["I"], case["J"]
        weights = I * J * esz // 2 + I * J // 8 if case["N"] <= 2 else I * J * esz
        nbytes = esz * T * (J + I) + weights + (esz * I if case["bias"] else 0) + (esz * T * I if case["residual"] else 0)
        if case["ckpt"]:                                                      # written, read and put back as values
            nbytes += 2 * ckpt(I) + esz * T * I
        return dict(bytes=nbytes, flops=2 * T * I * J * case["N"] // case["M"])
    if case["op"] == "checkpoint":
        return dict(bytes=2 * (esz * T * case["J"] + ckpt(case["J"])), flops=4 * T * case["J"])
    if case["op"] == "act_grad":
        return dict(bytes=2 * esz * T * case["I"] + ckpt(case["I"]) + 4 * case["I"], flops=10 * T * case["I"])
    I, J = case["I"], case["J"]
    return dict(bytes=esz * T * I + ckpt(J) + I * J * (4 if case["dw"] == "f32" else 2), flops=2 * T * I * J)


def _exact_kept(x):
    """What the checkpoint of rows in 64 bits stands for: the exponent by trial from the logarithm."""
    T, J = x.shape
    b = torch.zeros((T, -(-J // 32) * 32), dtype=torch.float64, device=x.device)
    b[:, :J] = x
    b = b.view(T, -1, 32)
    most = b.abs().max(dim=-1, keepdim=True).values
    e = torch.floor(torch.log2(most.clamp_min(2.0 ** -130))) - 8
    for _ in range(3):
        e = torch.where(torch.round(most * torch.exp2(-e)) > 127, e + 1, e)
    e = e.clamp(-126, 121)
    q = torch.round(b * torch.exp2(-e)).clamp(-127, 127)
    return (q * torch.exp2(e)).view(T, -1)[:, :J]


def exact(case, seed):
    state, op = prepare(case, seed), case["op"]
    half_erfc = lambda z: 0.5 * torch.special.erfc(-z / math.sqrt(2.0))  # noqa: E731
    tanh_arg = lambda z: math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)  # noqa: E731
    if op == "linear":
        z = torch.mm(state["X"].double(), state["W"].double().t())
        if case["bias"]:
            z += state["bias"].double()
        y = {"none": lambda: z, "relu": lambda: z.clamp_min(0.0), "gelu": lambda: z * half_erfc(z),
             "gelu_tanh": lambda: 0.5 * z * (1.0 + torch.tanh(tanh_arg(z))), "silu": lambda: z / (1.0 + torch.exp(-z))}[case["act"]]()
        if case["residual"]:
            y = y + state["residual"].double()
        return {"Y": y, "Z": _exact_kept(z)} if case["ckpt"] else {"Y": y}
    if op == "checkpoint":
        return {"X": _exact_kept(state["X"].double())}
    cols = case["I"] if op == "act_grad" else case["J"]
    T, blocks = case["T"], -(-cols // 32)
    scale = torch.exp2(state["ckpt"][T * blocks * 32:].double() - 127.0).view(T, blocks, 1)
    kept = (state["ckpt"][:T * blocks * 32].view(torch.int8).double().view(T, blocks, 32) * scale).view(T, -1)[:, :cols]
    if op == "weight_grad":
        return {"dW": torch.mm(state["dY"].double().t(), kept)}
    if case["act"] == "relu":
        slope = (kept > 0).double()
    elif case["act"] == "gelu":
        slope = half_erfc(kept) + kept * torch.exp(-kept ** 2 / 2.0) / math.sqrt(2.0 * math.pi)
    elif case["act"] == "gelu_tanh":
        t = torch.tanh(tanh_arg(kept))
        slope = 0.5 * (1.0 + t) + 0.5 * kept * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * kept ** 2)
    else:
        s = 1.0 / (1.0 + torch.exp(-kept))
        slope = s + kept * s * (1.0 - s)
    dZ = state["dY"].double() * slope
    return {"dZ": dZ, "dbias": dZ.sum(0)}
