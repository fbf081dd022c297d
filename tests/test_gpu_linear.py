"""The linear layer around the sparse product on the GPU: epilogue, 8-bit checkpoints, gradient through the activation, dense weight
gradient, against their definitions in 64 bits (linear_reference.py).

Sums of integers that fp32 holds exactly, in any order, are compared bit by bit; so are codes and scale bytes, which depend on their
inputs alone.  A rounding to the output's type is off by at most half a step, eps / 2 of the value."""
import numpy as np
import pytest

import linear_reference as ref
import oracle
import paper_2302_06058_amd as bm
from helpers import from_dev_f64, to_dev
from paper_2302_06058_amd import synth

pytestmark = pytest.mark.gpu
BF, F32 = synth.BF16, synth.F32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def tdt(dtype):
    import torch
    return torch.bfloat16 if dtype == BF else torch.float32


def rounded(a, dtype):
    """float64 -> the values that the stored type holds."""
    return synth.to_f64(synth.store(np.asarray(a, dtype=np.float32), dtype), dtype)


def dev(a, dtype):
    return to_dev(synth.store(np.asarray(a, dtype=np.float32), dtype), dtype)


def strided(a, dtype, pad, first=0, fill=0.0):
    """`a` as a view into a wider buffer, `first` elements in and with room for three more rows; returns (view, buffer)."""
    import torch
    T, C = a.shape
    buf = torch.full((first + (T + 3) * (C + pad),), fill, dtype=tdt(dtype), device="cuda")
    v = buf[first:first + T * (C + pad)].view(T, C + pad)[:, :C]
    v.copy_(dev(a, dtype))
    return v, buf


def ckpt_dev(codes, scales):
    import torch
    return torch.from_numpy(ref.join(codes, scales)).cuda()


# ---- checkpoints -----------------------------------------------------------------------------------------------------------------
def features(rng, T, C, dtype):
    x = rng.standard_normal((T, C)) * np.exp(rng.uniform(-20, 20, (T, 1)))
    x[rng.random((T, C)) < 0.02] = 0.0
    return rounded(x, dtype)


CKPT_SHAPES = [(1, 1), (1, 31), (1, 33), (3, 32), (5, 147), (64, 64), (130, 1000), (7, 4099), (2, 11008), (3001, 48)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,C", CKPT_SHAPES)
@pytest.mark.parametrize("pad,first", [(0, 0), (8, 0), (3, 1)])
def test_checkpoint_is_the_rule_bit_by_bit(T, C, dtype, pad, first):
    import torch
    rng = np.random.default_rng(T * 7919 + C)
    x = features(rng, T, C, dtype)
    X, _ = strided(x, dtype, pad, first, float("nan"))                 # what lies beside the rows is no part of them
    n = bm.checkpoint_bytes(T, C)
    buf = torch.full((n + 64,), 77, dtype=torch.uint8, device="cuda")
    assert bm.bimask_checkpoint_store(X, buf[:n]).data_ptr() == buf.data_ptr()
    got = buf.cpu().numpy()
    assert (got[n:] == 77).all()
    codes, scales = ref.store(x)
    gc, gs = ref.split(got[:n], T, C)
    live = np.abs(codes.reshape(T, -1, 32)).max(-1) > 0                # (a block of zeros has any scale)
    assert (gc == codes).all() and (gs == scales)[live].all()
    out, whole = strided(np.full((T, C), 5.0), dtype, pad, first, 5.0)
    bm.bimask_checkpoint_load(buf[:n], T, C, X=out)
    assert (from_dev_f64(out, dtype) == ref.load(codes, scales, C)).all()
    out.fill_(5.0)
    assert (whole == 5.0).all(), "written beside or behind the rows"
    assert torch.equal(bm.bimask_checkpoint_load(buf[:n], T, C, tdt(dtype)), bm.bimask_checkpoint_load(buf[:n], T, C, torch.float32).to(tdt(dtype)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_checkpoint_of_extreme_blocks(dtype):
    big, tiny = (3.3895313892515355e38, 9.183549615799121e-41) if dtype == BF else (3.4028234663852886e38, 1.401298464324817e-45)
    rows = [np.zeros(32), -np.zeros(32), np.full(32, big), np.full(32, -big), np.full(32, tiny), np.full(32, 2.0 ** -126), np.full(32, 127 * 2.0 ** -126),
            np.full(32, 128 * 2.0 ** -126)]
    for m in (126.5, 127.0, 127.5, 128.0, 1.0, 63.5, 64.0, 255 / 128):                  # at and around the borders of a power
        for k in (0, 7, -120, 60):
            r = np.linspace(-1, 1, 32) * m * 2.0 ** k
            r[5] = m * 2.0 ** k
            rows.append(r)
    bad = []
    for v in (np.inf, -np.inf, np.nan):
        r = np.arange(32.0)
        r[17] = v
        bad.append(r)
    x = rounded(np.stack(rows + bad), dtype)
    codes, scales = ref.store(x)
    ck = bm.bimask_checkpoint_store(dev(x, dtype))
    gc, gs = ref.split(ck.cpu().numpy(), *x.shape)
    live = np.abs(codes).max(-1, keepdims=True) > 0
    assert (gc == codes).all() and (gs == scales)[live | (scales == 255)].all()
    out = from_dev_f64(bm.bimask_checkpoint_load(ck, *x.shape, tdt(dtype)), dtype)
    want = ref.load(codes, scales, 32)
    assert np.array_equal(out, want, equal_nan=True) and np.isnan(out[-3:]).all() and np.isfinite(out[:-3]).all()
    step = 2.0 ** (scales.astype(np.float64) - 127)
    off = np.abs(want - x)[:-3] / step[:-3]
    # half a step; where e is kept to 121, |x| < 2^128 is below 128 steps and clamped to 127: less than a whole one
    assert off.max() < 1.0 and off[4:].max() <= 0.5


# ---- product with its epilogue ------------------------------------------------------------------------------------------------------
def masked_integers(rng, I, J, N, M):
    W = rng.integers(1, 8, (I, J)) * rng.choice((-1, 1), (I, J)).astype(np.float64)
    B = oracle.forward_mask(W, N, M)
    return W, W * B


def few_ones(rng, T, J):
    """Token rows with four non-zeros +-1, so that sums stay within 4 * 7."""
    x = np.zeros((T, J))
    for _ in range(4):
        x[np.arange(T), rng.integers(0, J, T)] = rng.choice((-1.0, 1.0), T)
    return x


def operand(W, N, M, dtype):
    _, v, x = bm.bimask_forward_mask_compress(dev(W, dtype), N, M)
    return v, x


# (I, J, T, N, M, type, extra columns of X / Y / residual): every form of every kernel (a host test holds the list to that)
LINEAR = [
    (32, 64, 1, 2, 4, BF, 0), (36, 72, 7, 1, 4, BF, 0), (64, 4096, 32, 2, 4, BF, 0), (100, 1100, 5, 2, 4, BF, 0), (48, 136, 31, 4, 8, BF, 0), (1000, 2048, 3, 2, 4, BF, 6),
    (40, 2056, 17, 4, 8, BF, 2), (4100, 132, 1, 2, 4, BF, 0),
    (64, 384, 100, 2, 4, BF, 0), (512, 264, 64, 2, 4, BF, 0), (512, 388, 64, 2, 4, BF, 2), (64, 256, 784, 4, 8, BF, 0), (136, 640, 60, 4, 8, BF, 0), (136, 648, 60, 4, 8, BF, 0),
    (136, 648, 60, 4, 8, BF, 2), (64, 128, 1000, 2, 4, BF, 0), (64, 136, 9000, 2, 4, BF, 0), (60, 132, 900, 2, 4, BF, 2), (64, 128, 8200, 4, 8, BF, 0), (64, 136, 1000, 4, 8, BF, 0),
    (64, 136, 1000, 4, 8, BF, 2), (384, 256, 2000, 2, 4, BF, 0), (384, 200, 2000, 2, 8, BF, 0), (388, 260, 700, 2, 4, BF, 2), (384, 256, 2000, 4, 8, BF, 0), (384, 200, 2000, 4, 8, BF, 0),
    (384, 200, 700, 4, 8, BF, 2), (1024, 128, 6200, 2, 4, BF, 0), (1008, 136, 6200, 2, 4, BF, 0), (1008, 132, 6200, 2, 4, BF, 2), (1024, 128, 6200, 4, 8, BF, 0), (1008, 136, 6200, 4, 8, BF, 0),
    (1008, 136, 6200, 4, 8, BF, 2), (1024, 640, 6200, 2, 4, BF, 0), (1008, 648, 6200, 2, 4, BF, 0), (1024, 640, 6200, 4, 8, BF, 0), (1008, 648, 6200, 4, 8, BF, 0),
    (64, 2176, 3, 2, 4, BF, 0), (100, 2184, 13, 2, 4, BF, 0), (100, 2184, 20, 2, 4, BF, 0), (4100, 2180, 20, 1, 4, BF, 2), (4100, 2184, 37, 2, 4, BF, 0), (512, 384, 1100, 2, 4, BF, 0),
    (512, 392, 1100, 2, 4, BF, 0), (512, 388, 1100, 2, 4, BF, 2), (512, 384, 25211, 2, 4, BF, 0), (520, 384, 25211, 4, 8, BF, 8), (192, 384, 1, 1, 16, BF, 0),
    (64, 128, 32, 2, 4, F32, 0), (16, 32, 5, 1, 4, F32, 0), (36, 64, 33, 2, 4, F32, 1), (48, 300, 70, 2, 4, F32, 0), (48, 32, 5, 4, 8, F32, 0), (40, 64, 5, 4, 8, F32, 3), (72, 128, 50, 4, 8, F32, 0),
    (72, 400, 50, 4, 8, F32, 0), (256, 32, 32777, 2, 4, F32, 0), (256, 64, 8200, 2, 4, F32, 0), (260, 128, 8200, 2, 4, F32, 0), (256, 32, 32777, 4, 8, F32, 0), (256, 64, 8200, 4, 8, F32, 0),
    (264, 128, 8200, 4, 8, F32, 0)]
# large sizes of the bf16 product, checked against the plain product of the library on the same operands
LARGE = [(4096, 1152, 8200, 2, 4), (2048, 2048, 16500, 1, 4)]


@pytest.mark.parametrize("I,J,T,N,M,dtype,pad", LINEAR)
def test_linear_sums_are_exact_with_bias_residual_and_checkpoint(I, J, T, N, M, dtype, pad):
    import torch
    rng = np.random.default_rng(I * 131 + J * 17 + T)
    W, Wm = masked_integers(rng, I, J, N, M)
    x, bias, res = few_ones(rng, T, J), rng.integers(-20, 21, I).astype(np.float64), rng.integers(-60, 61, (T, I)).astype(np.float64)
    z = x @ Wm.T + bias                                                # within 28 + 20
    X, _ = strided(x, dtype, pad, 0, float("nan"))
    R, _ = strided(res, dtype, pad)
    Y, whole = strided(np.full((T, I), 99.0), dtype, pad, 0, 99.0)
    v, idx = operand(W, N, M, dtype)
    out, ck = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=dev(bias[None], dtype)[0], residual=R, Y=Y, want_ckpt=True)
    assert out is Y
    assert (from_dev_f64(Y, dtype) == z + res).all()
    codes, scales = ref.store(z)
    gc, gs = ref.split(ck.cpu().numpy(), T, I)
    live = np.abs(codes.reshape(T, -1, 32)).max(-1) > 0
    assert (gc == codes).all() and (gs == scales)[live].all()
    Y.fill_(99.0)
    assert (whole == 99.0).all(), "written beside or behind the rows"
    # without anything, and the relu: exact as well; in place on the residual
    assert (from_dev_f64(bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M)[0], dtype) == x @ Wm.T).all()
    bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=dev(bias[None], dtype)[0], act=bm.ACT_RELU, residual=R, Y=R)
    assert (from_dev_f64(R, dtype) == np.maximum(z, 0.0) + res).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("a", ref.ACTS)
@pytest.mark.parametrize("I,J,T,N,M,dtype", [(100, 1100, 5, 2, 4, BF), (64, 384, 100, 2, 4, BF), (384, 200, 700, 4, 8, BF), (1024, 128, 6200, 2, 4, BF), (48, 300, 70, 2, 4, F32), (256, 64, 8200, 4, 8, F32)])
def test_linear_activations(I, J, T, N, M, dtype, a):
    rng = np.random.default_rng(I + J + T)
    W = rounded(rng.standard_normal((I, J)) * 2.0 / np.sqrt(J * N / M), dtype)
    B = oracle.forward_mask(W, N, M)
    x, bias, res = (rounded(rng.standard_normal(s), dtype) for s in ((T, J), (I,), (T, I)))
    z = x @ (W * B).T + bias
    v, idx = operand(W, N, M, dtype)
    Y, ck = bm.bimask_sparse_linear_fwd(dev(x, dtype), v, idx, I, J, N, M, bias=dev(bias[None], dtype)[0], act=bm.ACTS[a], residual=dev(res, dtype), want_ckpt=True)
    want = ref.act(z, a) + res
    dz = (J + 2) * 2.0 ** -24 * (np.abs(x) @ np.abs(W * B).T + np.abs(bias))           # J products and two sums in fp32
    off = 1.13 * dz + ref.function_error(z, a) * np.abs(ref.act(z, a)) + 2.0 ** -24 * np.abs(want)      # no slope exceeds 1.13
    off += ref.coarse_gelu(z, a) if dtype == BF else 0.0
    assert (np.abs(from_dev_f64(Y, dtype) - want) <= HALF[dtype] * np.abs(want) + 1.01 * off).all()
    # the checkpoint is off from Z by half a step of its block and what Z itself is off
    codes, scales = ref.split(ck.cpu().numpy(), T, I)
    step = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=1)[:, :I]
    assert (np.abs(ref.load(codes, scales, I) - z) <= 0.5 * step + dz).all()


@pytest.mark.parametrize("I,J,T,N,M", LARGE)
def test_large_linear_is_the_plain_product_of_the_library(I, J, T, N, M):
    import torch
    g = torch.Generator(device="cuda").manual_seed(I + T)
    W = torch.randn((I, J), device="cuda", generator=g).mul_(0.02).bfloat16()
    X, R = (torch.randn((T, n), device="cuda", generator=g).bfloat16() for n in (J, I))
    bias = torch.randn((I,), device="cuda", generator=g).bfloat16()
    _, v, idx = bm.bimask_forward_mask_compress(W, N, M)
    got, _ = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M)
    plain = bm.bimask_sparse_gemm_fwd(X, v, idx, I, J, N, M)
    # the two round sums that differ by the order of additions: rarely another neighbour, never more
    assert ((got.float() - plain.float()).abs() <= 2.0 ** -7 * plain.float().abs() + 1e-4).all()
    Y, ck = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=bias, act=bm.ACT_SILU, residual=R, want_ckpt=True)
    z = plain.double() + bias.double()                                  # plain is off by half a step of bf16
    want = z * torch.sigmoid(z) + R.double()
    assert ((Y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.1 * 2.0 ** -8 * plain.double().abs() + 1e-4).all()
    Z = bm.bimask_checkpoint_load(ck, T, I, torch.float32).double()
    most = torch.nn.functional.pad(z, (0, -I % 32)).view(T, -1, 32).abs().amax(-1, keepdim=True).expand(-1, -1, 32).reshape(T, -1)[:, :I]
    assert ((Z - z).abs() <= most / 127 + 2.0 ** -8 * plain.double().abs() + 1e-4).all()      # half a step is at most max / 127.5
    assert torch.equal(bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=bias, act=bm.ACT_SILU, residual=R)[0], Y)


def test_padding_features_and_masked_tokens_stay_out_of_the_checkpoint():
    """A token with an infinity makes its own blocks NaN and no other token's; features beyond I count as 0."""
    I, J = 36, 64
    rng = np.random.default_rng(3)
    W, Wm = masked_integers(rng, I, J, 2, 4)
    for T, dtype in ((5, BF), (70, BF), (5, F32)):
        x = few_ones(rng, T, J)
        v, idx = operand(W, 2, 4, dtype)
        clean = bm.bimask_sparse_linear_fwd(dev(x, dtype), v, idx, I, J, 2, 4, want_ckpt=True)[1]
        x[3] = np.inf
        ck = bm.bimask_sparse_linear_fwd(dev(x, dtype), v, idx, I, J, 2, 4, want_ckpt=True)[1]
        Z = from_dev_f64(bm.bimask_checkpoint_load(ck, T, I, tdt(dtype)), dtype)
        Zc = from_dev_f64(bm.bimask_checkpoint_load(clean, T, I, tdt(dtype)), dtype)
        assert np.isnan(Z[3]).all()
        keep = np.arange(T) != 3
        assert (Z[keep] == Zc[keep]).all()


# ---- gradient through the activation -------------------------------------------------------------------------------------------------
ACT_SHAPES = [(1, 1), (1, 33), (7, 16), (130, 1000), (4097, 40), (33, 11008), (1000, 147), (70000, 16)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("a", ref.ACTS)
@pytest.mark.parametrize("T,I", ACT_SHAPES)
def test_act_bwd(T, I, a, dtype):
    import torch
    rng = np.random.default_rng(T + I)
    codes, scales = ref.store(rng.standard_normal((T, I)) * np.exp(rng.uniform(-3, 3, (T, 1))))
    dy = rounded(rng.standard_normal((T, I)), dtype)
    z = ref.load(codes, scales, I)
    want, err = dy * ref.slope(z, a), np.abs(dy) * (ref.slope_error(z, a) + 2.0 ** -24 * np.abs(ref.slope(z, a)))
    for pad, first in ((0, 0), (5, 1)):
        D, _ = strided(dy, dtype, pad, first, float("nan"))
        dZ, whole = strided(np.full((T, I), 9.0), dtype, pad, first, 9.0)
        ck = ckpt_dev(codes, scales)
        out, db = bm.bimask_act_bwd(D, ck, bm.ACTS[a], dZ=dZ)
        assert out is dZ and db.dtype == torch.float32
        got = from_dev_f64(dZ, dtype)
        assert (np.abs(got - want) <= HALF[dtype] * np.abs(want) + 1.01 * err).all()
        bound = err.sum(0) + T * 2.0 ** -24 * np.abs(want).sum(0)                       # T additions in fp32, any order
        assert (np.abs(from_dev_f64(db, F32) - want.sum(0)) <= 1.01 * bound).all()
        alone = bm.bimask_act_bwd(D, ck, bm.ACTS[a], want_dZ=False)[1]
        assert torch.equal(alone, db)
        nothing, none = bm.bimask_act_bwd(D, ck, bm.ACTS[a], want_dbias=False)
        assert none is None and torch.equal(nothing, dZ)
        if a == "none":
            assert torch.equal(bm.bimask_act_bwd(D, None, bm.ACT_NONE, want_dZ=False)[1], db)
        bm.bimask_act_bwd(D, ck, bm.ACTS[a], dZ=D, want_dbias=False)                    # in place
        assert torch.equal(D, dZ)
        dZ.fill_(9.0)
        assert (whole == 9.0).all(), "written beside or behind the rows"


@pytest.mark.parametrize("a", ref.ACTS[1:])
def test_slopes_at_the_ends_and_against_differences(a):
    """The slope over the whole range of a checkpoint (codes +-127 at powers from 2^-20 to 2^100), and against differences of the
    activation in 64 bits: (f(z + h) - f(z - h)) / 2h is off by h^2 / 6 f''' (below 2 h^2) and 2^-52 |f| / h."""
    scales = np.arange(107, 228, dtype=np.uint8)[:, None]
    codes = np.tile(np.array([-127, -126, -100, -64, -63, -17, -9, -5, -3, -2, -1, 0, 1, 2, 3, 5, 9, 17, 33, 63, 64, 65, 90, 100, 101, 110, 120, 122, 124, 125, 126, 127], dtype=np.int8), (len(scales), 1))
    z = ref.load(codes, scales, 32)
    got = from_dev_f64(bm.bimask_act_bwd(dev(np.ones_like(z), F32), ckpt_dev(codes, scales), bm.ACTS[a], want_dbias=False)[0], F32)
    want = ref.slope(np.clip(z, -700, 700), a)                         # (flat beyond; the reference's powers are not)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 1.01 * ref.slope_error(np.clip(z, -700, 700), a)).all()
    near, h = np.abs(z) < 20, 1e-5
    if a == "relu":
        near &= np.abs(z) > h
    zn = z[near]
    d = (ref.act(zn + h, a) - ref.act(zn - h, a)) / (2 * h)
    assert (np.abs(got[near] - d) <= 2 * h * h + 2.0 ** -50 * (1 + np.abs(zn)) / h + 2.0 ** -22 + 1.01 * ref.slope_error(zn, a)).all()


def test_not_a_number_in_a_checkpoint_reaches_the_gradient():
    codes, scales = ref.store(np.ones((4, 64)))
    scales[2, 1] = 255
    for a in ref.ACTS[1:]:
        dZ, db = bm.bimask_act_bwd(dev(np.ones((4, 64)), BF), ckpt_dev(codes, scales), bm.ACTS[a])
        bad = np.isnan(from_dev_f64(dZ, BF))
        assert bad[2, 32:].all() and bad.sum() == 32 and np.isnan(from_dev_f64(db, F32)[32:]).all() and np.isfinite(from_dev_f64(db, F32)[:32]).all()


# ---- weight gradient ------------------------------------------------------------------------------------------------------------------
# (I, J, T, type of dY, type of dW, extra columns): every form of every kernel
GRADS = [(1, 1, 1, BF, BF, 0), (8, 16, 3, BF, F32, 0), (33, 147, 65, BF, BF, 0), (64, 576, 5000, BF, F32, 0), (128, 128, 64, BF, BF, 8), (130, 1000, 257, BF, F32, 3), (1000, 72, 700, BF, BF, 0),
         (4096, 3336, 96, BF, BF, 0), (4097, 3300, 130, BF, F32, 1), (64, 148, 20011, BF, BF, 0), (1000, 40, 700, BF, BF, 0), (301, 64, 9000, BF, F32, 1), (5, 300, 9000, BF, F32, 0), (15, 65, 33, BF, BF, 0), (40, 500, 300, BF, BF, 0), (505, 512, 49999, BF, F32, 0), (1031, 131, 5000, BF, BF, 0), (1, 3, 9000, BF, F32, 0), (3, 1, 20000, F32, F32, 0), (8, 300, 31, BF, BF, 1), (1, 1, 1, F32, F32, 0), (65, 130, 40, F32, F32, 0), (64, 128, 32, F32, F32, 4), (200, 96, 3000, F32, F32, 1),
         (4360, 4090, 770, BF, F32, 1), (4100, 4096, 770, BF, BF, 0), (2060, 8200, 800, BF, BF, 0)]      # whole rounds of large tiles, the rows behind them in a second launch


@pytest.mark.parametrize("I,J,T,dtype,dw,pad", GRADS)
def test_weight_grad_sums_are_exact(I, J, T, dtype, dw, pad):
    import torch
    rng = np.random.default_rng(I * 31 + J * 7 + T)
    dy, x = rng.integers(-2, 3, (T, I)).astype(np.float64), rng.integers(-3, 4, (T, J)).astype(np.float64)
    D, _ = strided(dy, dtype, pad, 1 if pad % 2 else 0, float("nan"))
    ck = bm.bimask_checkpoint_store(dev(x, dtype))
    want = dy.T @ x                                                    # within 6 T < 2^24: exact in fp32 in any order
    dW, whole = strided(np.full((I, J), 7.0), dw, pad, 0, 7.0)
    assert bm.bimask_weight_grad(D, ck, J, dW=dW) is dW
    assert (from_dev_f64(dW, dw) == rounded(want, dw)).all()
    old = rounded(want, dw)
    bm.bimask_weight_grad(D, ck, J, dW=dW, accumulate=True)
    assert (from_dev_f64(dW, dw) == rounded(want + old, dw)).all()
    assert torch.equal(bm.bimask_weight_grad(D, ck, J, dw_dtype=tdt(dw)), dev(want, dw))
    dW.fill_(7.0)
    assert (whole == 7.0).all(), "written beside or behind the rows"


@pytest.mark.parametrize("I,J,T,dtype", [(64, 576, 5000, BF), (300, 200, 9000, BF), (200, 96, 3000, F32), (4096, 3336, 2000, BF)])
def test_weight_grad_of_reals(I, J, T, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(T)
    dY = torch.randn((T, I), device="cuda", generator=g).to(tdt(dtype))
    ck = bm.bimask_checkpoint_store(torch.randn((T, J), device="cuda", generator=g).to(tdt(dtype)))
    X = bm.bimask_checkpoint_load(ck, T, J, tdt(dtype)).double()
    got = bm.bimask_weight_grad(dY, ck, J, dw_dtype=torch.float32)
    want, mass = dY.double().t() @ X, dY.double().abs().t() @ X.abs()
    assert ((got.double() - want).abs() <= T * 2.0 ** -24 * mass).all()
    assert torch.equal(bm.bimask_weight_grad(dY, ck, J, dw_dtype=torch.float32), got)       # the same bits again


def test_not_a_number_and_infinity_reach_the_weight_gradient_and_their_rows_only():
    T, I, J = 70, 40, 96
    rng = np.random.default_rng(9)
    dy, x = rng.integers(-2, 3, (T, I)).astype(np.float64), rng.integers(1, 4, (T, J)).astype(np.float64)
    dy[5, 3] = np.inf
    x[66, 40] = np.nan                                                 # the block 32 .. 63 of token 66
    dW = from_dev_f64(bm.bimask_weight_grad(dev(dy, BF), bm.bimask_checkpoint_store(dev(x, BF)), J, dw_dtype=tdt(F32)), F32)
    assert np.isnan(dW[:, 32:64]).all() and np.isposinf(dW[3, :32]).all() and np.isposinf(dW[3, 64:]).all()
    rest = np.delete(np.delete(dW, 3, 0), np.s_[32:64], 1)
    keep = [i for i in range(I) if i != 3]
    assert (rest == (dy[:, keep].T @ np.nan_to_num(x))[:, list(range(32)) + list(range(64, 96))]).all()


# ---- together --------------------------------------------------------------------------------------------------------------------------
def mlp_buffers(rng, I, J, T, dtype, N=2, M=4):
    b = {}
    for name, (o, i) in (("up", (I, J)), ("down", (J, I))):
        W = dev(rng.standard_normal((o, i)) / np.sqrt(i * N / M), dtype)
        B, v, x = bm.bimask_forward_mask_compress(W, N, M)
        P = to_i32(rng.permutation(o))
        _, vb, xb = bm.bimask_backward_mask_compress(W, N, M, B, P)
        b[name] = dict(W=W, v=v, x=x, vb=vb, xb=xb, P=P, bias=dev(rng.standard_normal((1, o)), dtype)[0])
    return b


def to_i32(a):
    import torch
    return torch.from_numpy(a.astype(np.int32)).cuda()


def mlp_step(b, X, dY, I, J, a, N=2, M=4):
    """One training step of X + down(act(up(X))): outputs and gradients, everything that crosses to the backward pass in 8 bits."""
    T = X.shape[0]
    u, d = b["up"], b["down"]
    kX = bm.bimask_checkpoint_store(X)
    H, kZ = bm.bimask_sparse_linear_fwd(X, u["v"], u["x"], I, J, N, M, bias=u["bias"], act=bm.ACTS[a], want_ckpt=True)
    kH = bm.bimask_checkpoint_store(H)
    Y, _ = bm.bimask_sparse_linear_fwd(H, d["v"], d["x"], J, I, N, M, bias=d["bias"], residual=X)
    dWd, dbd = bm.bimask_weight_grad(dY, kH, I), bm.bimask_act_bwd(dY, None, bm.ACT_NONE, want_dZ=False)[1]
    dH = bm.bimask_sparse_gemm_bwd(dY, d["P"], d["vb"], d["xb"], J, I, N, M)
    dZ, dbu = bm.bimask_act_bwd(dH, kZ, bm.ACTS[a])
    dWu = bm.bimask_weight_grad(dZ, kX, J)
    dX = bm.bimask_sparse_gemm_bwd(dZ, u["P"], u["vb"], u["xb"], I, J, N, M)
    return dict(H=H, Y=Y, dWd=dWd, dbd=dbd, dH=dH, dZ=dZ, dbu=dbu, dWu=dWu, dX=dX, kX=kX, kZ=kZ, kH=kH, X=X, dY=dY)


@pytest.mark.parametrize("I,J,T,a,dtype", [(256, 128, 100, "gelu", BF), (512, 136, 1000, "silu", BF), (128, 64, 37, "gelu_tanh", F32), (1536, 384, 394, "gelu", BF)])
def test_training_step_of_an_mlp_block(I, J, T, a, dtype):
    """Each call against its formula, on what the calls before it gave."""
    rng = np.random.default_rng(I + T)
    b = mlp_buffers(rng, I, J, T, dtype)
    r = mlp_step(b, dev(rng.standard_normal((T, J)), dtype), dev(rng.standard_normal((T, J)), dtype), I, J, a)
    h = {k: from_dev_f64(r[k], dtype) for k in ("X", "dY", "H", "Y", "dH", "dZ", "dWd", "dWu")}
    kX, kZ, kH = (ref.load(*ref.split(r[k].cpu().numpy(), T, C), C) for k, C in (("kX", J), ("kZ", I), ("kH", I)))
    masked = {k: from_dev_f64(b[k]["W"], dtype) * oracle.forward_mask(from_dev_f64(b[k]["W"], dtype), 2, 4) for k in b}
    bias = {k: from_dev_f64(b[k]["bias"], dtype) for k in b}
    half, ulp = HALF[dtype], 2.0 ** -24
    z = h["X"] @ masked["up"].T + bias["up"]
    dz = (J + 2) * ulp * (np.abs(h["X"]) @ np.abs(masked["up"]).T + np.abs(bias["up"]))
    want = ref.act(z, a)
    assert (np.abs(h["H"] - want) <= half * np.abs(want) + 1.14 * dz + ref.function_error(z, a) * np.abs(want) + (ref.coarse_gelu(z, a) if dtype == BF else 0.0)).all()
    assert np.abs(kX - h["X"]).max() <= np.abs(h["X"]).max() / 127 and np.abs(kH - h["H"]).max() <= np.abs(h["H"]).max() / 127
    want = h["H"] @ masked["down"].T + bias["down"] + h["X"]
    assert (np.abs(h["Y"] - want) <= half * np.abs(want) + (I + 3) * ulp * (np.abs(h["H"]) @ np.abs(masked["down"]).T + np.abs(bias["down"]) + np.abs(h["X"]))).all()
    want = h["dH"] * ref.slope(kZ, a)
    err = np.abs(h["dH"]) * (ref.slope_error(kZ, a) + ulp * np.abs(ref.slope(kZ, a)))
    assert (np.abs(h["dZ"] - want) <= half * np.abs(want) + 1.01 * err).all()
    assert (np.abs(from_dev_f64(r["dbu"], F32) - want.sum(0)) <= 1.01 * err.sum(0) + T * ulp * np.abs(want).sum(0)).all()
    assert (np.abs(from_dev_f64(r["dbd"], F32) - h["dY"].sum(0)) <= T * ulp * np.abs(h["dY"]).sum(0)).all()
    for g, D, x in (("dWd", h["dY"], kH), ("dWu", h["dZ"], kX)):
        want = D.T @ x
        assert (np.abs(h[g] - want) <= half * np.abs(want) + T * ulp * (np.abs(D).T @ np.abs(x))).all()


def test_gradients_against_differences_of_the_loss():
    """Integers that a checkpoint holds exactly: loss(W, b) = sum G * gelu(X W^T + b), differences in 64 bits against the two calls."""
    rng = np.random.default_rng(5)
    T, I, J = 40, 8, 16
    x, W, bias = rng.integers(-1, 2, (T, J)).astype(float), rng.integers(-1, 2, (I, J)) / 4.0, rng.integers(-2, 3, I) / 4.0
    G = rounded(rng.standard_normal((T, I)), F32)
    z = x @ W.T + bias                                                 # quarters, within 4.5: 18 steps
    kZ, kX = bm.bimask_checkpoint_store(dev(z, F32)), bm.bimask_checkpoint_store(dev(x, F32))
    assert (from_dev_f64(bm.bimask_checkpoint_load(kZ, T, I, tdt(F32)), F32) == z).all()
    dZ, db = bm.bimask_act_bwd(dev(G, F32), kZ, bm.ACT_GELU)
    dW = from_dev_f64(bm.bimask_weight_grad(dZ, kX, J), F32)
    loss = lambda W, b: (G * ref.act(x @ W.T + b, "gelu")).sum()  # noqa: E731
    h = 1e-5
    # truncation: h^2 / 6 times third derivatives (below 2) over T terms; rounding of the loss: 2^-50 / h of its size; the calls: fp32
    mass = np.abs(G).sum() * 6
    tol = 2 * h * h * mass + 2.0 ** -50 * mass / h + T * 2.0 ** -19 * np.abs(G).sum(0).max()
    for i in range(I):
        e = np.zeros(I)
        e[i] = h
        assert abs(from_dev_f64(db, F32)[i] - (loss(W, bias + e) - loss(W, bias - e)) / (2 * h)) <= tol
        for j in range(0, J, 5):
            E = np.zeros((I, J))
            E[i, j] = h
            assert abs(dW[i, j] - (loss(W + E, bias) - loss(W - E, bias)) / (2 * h)) <= tol


def test_a_captured_step_replays_as_the_eager_one():
    """All calls of a step in one graph (two kernels for the bias gradient and for split weight gradients), replayed on new inputs with
    eager work between the replays; and on a stream of its own."""
    import torch
    rng = np.random.default_rng(11)
    I, J, T = 256, 128, 3000
    b = mlp_buffers(rng, I, J, T, BF)
    X, dY = dev(rng.standard_normal((T, J)), BF), dev(rng.standard_normal((T, J)), BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = mlp_step(b, X, dY, I, J, "silu")
    torch.cuda.current_stream().wait_stream(side)
    keys = ("H", "Y", "dWd", "dbd", "dZ", "dbu", "dWu", "dX", "kX", "kZ", "kH")
    eager = mlp_step(b, X, dY, I, J, "silu")
    assert all(torch.equal(first[k], eager[k]) for k in keys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mlp_step(b, X, dY, I, J, "silu")
    for seed in range(4):
        rng = np.random.default_rng(seed)
        X.copy_(dev(rng.standard_normal((T, J)), BF))
        dY.copy_(dev(rng.standard_normal((T, J)), BF))
        graph.replay()
        got = {k: out[k].clone() for k in keys}
        want = mlp_step(b, X, dY, I, J, "silu")
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in keys), (seed, [k for k in keys if not torch.equal(got[k], want[k])])


def test_single_rows_and_columns_of_other_layouts():
    """A single token whatever its strides say, a view of every other row, a matrix of one column."""
    import torch
    rng = np.random.default_rng(2)
    W, Wm = masked_integers(rng, 32, 64, 2, 4)
    v, idx = operand(W, 2, 4, BF)
    x = few_ones(rng, 6, 64)
    X = dev(x, BF)
    row = X[2].clone().unsqueeze(1).t()                                # shape (1, 64), strides (1, 1)
    assert row.stride() == (1, 1)
    assert (from_dev_f64(bm.bimask_sparse_linear_fwd(row, v, idx, 32, 64, 2, 4)[0], BF) == x[2:3] @ Wm.T).all()
    assert (from_dev_f64(bm.bimask_sparse_linear_fwd(X[::2], v, idx, 32, 64, 2, 4)[0], BF) == x[::2] @ Wm.T).all()
    col = dev(rng.integers(-3, 4, (9, 4)).astype(float), F32)[:, 1:2]
    assert torch.equal(bm.bimask_checkpoint_load(bm.bimask_checkpoint_store(col), 9, 1, torch.float32), col)


def test_outputs_stay_within_checkpoint_and_workspace():
    """Bytes behind a checkpoint that the product writes, and behind workspaces, stay as they were."""
    import torch
    rng = np.random.default_rng(7)
    for I, J, T, dtype in ((36, 64, 5, BF), (100, 1100, 37, BF), (1008, 136, 6200, BF), (40, 64, 5, F32)):
        W, _ = masked_integers(rng, I, J, 2, 4)
        v, idx = operand(W, 2, 4, dtype)
        n = bm.checkpoint_bytes(T, I)
        buf = torch.full((n + 256,), 99, dtype=torch.uint8, device="cuda")
        X = dev(few_ones(rng, T, J), dtype)
        Y, ck = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, 2, 4, ckpt=buf[:n])
        assert ck.data_ptr() == buf.data_ptr() and (buf[n:] == 99).all()
        assert torch.equal(ck, bm.bimask_sparse_linear_fwd(X, v, idx, I, J, 2, 4, want_ckpt=True)[1])
    for I, J, T in ((64, 576, 5000), (300, 200, 9000), (512, 512, 49999)):
        for kind, call in ((bm.WS_ACT_BWD, lambda ws: bm.bimask_act_bwd(dY, None, bm.ACT_NONE, want_dZ=False, workspace=ws)[1]), (bm.WS_WEIGHT_GRAD, lambda ws: bm.bimask_weight_grad(dY, ck, J, workspace=ws))):
            dY = dev(rng.integers(-2, 3, (T, I)).astype(float), BF)
            ck = bm.bimask_checkpoint_store(dev(rng.integers(-2, 3, (T, J)).astype(float), BF))
            need = bm.workspace_bytes(kind, I, J, T, 0, bm.BF16, 0, 0)
            assert need > 0
            buf = torch.full((need + 256,), 99, dtype=torch.uint8, device="cuda")
            assert torch.equal(call(buf[:need]), call(None)) and (buf[need:] == 99).all()


def test_two_steps_at_once_on_two_streams():
    """Calls on two streams share nothing: the same bits as one after the other."""
    import torch
    rng = np.random.default_rng(23)
    I, J, T = 512, 256, 2000
    b = mlp_buffers(rng, I, J, T, BF)
    xs = [(dev(rng.standard_normal((T, J)), BF), dev(rng.standard_normal((T, J)), BF)) for _ in range(2)]
    want = [mlp_step(b, X, dY, I, J, "gelu_tanh") for X, dY in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(3):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(mlp_step(b, *xs[k], I, J, "gelu_tanh"))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(g[n], want[k][n]) for n in ("H", "Y", "dWd", "dbd", "dZ", "dbu", "dWu", "dX", "kZ"))


def test_infinities_and_nan_of_a_token_stay_with_it():
    """Activations of infinite and NaN sums; other tokens keep their bits, in every kernel form that bf16 has."""
    import torch
    rng = np.random.default_rng(29)
    for I, J, T, N, M in ((64, 4096, 4, 2, 4), (512, 264, 64, 2, 4), (64, 128, 1000, 2, 4), (1008, 136, 6200, 2, 4), (384, 200, 700, 4, 8)):
        W, _ = masked_integers(rng, I, J, N, M)
        v, idx = operand(np.abs(W), N, M, BF)
        X = dev(few_ones(rng, T, J), BF)
        for a, at_inf in (("relu", np.inf), ("gelu", np.inf), ("gelu_tanh", np.inf), ("silu", np.inf), ("none", np.inf)):
            clean = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, act=bm.ACTS[a])[0]
            D = X.clone()
            D[1], D[2] = 3e38, float("nan")                            # sums of like signs beyond bf16 and fp32: +inf
            Y = bm.bimask_sparse_linear_fwd(D, v, idx, I, J, N, M, act=bm.ACTS[a])[0]
            assert (Y[1] == at_inf).all() and torch.isnan(Y[2]).all(), (a, I)
            keep = [t for t in range(T) if t not in (1, 2)]
            assert torch.equal(Y[keep], clean[keep]), (a, I)


def test_wrappers_refuse_what_does_not_fit():
    """Types, sizes and layouts that the wrappers or the library refuse, and nothing is launched."""
    import torch
    rng = np.random.default_rng(31)
    W, _ = masked_integers(rng, 64, 128, 2, 4)
    v, idx = operand(W, 2, 4, BF)
    X, R = dev(few_ones(rng, 6, 128), BF), dev(np.ones((6, 64)), BF)
    f = lambda **k: bm.bimask_sparse_linear_fwd(**{**dict(X=X, Wf_values=v, Wf_index=idx, I=64, J=128, N=2, M=4), **k})  # noqa: E731
    f()
    for bad in (dict(J=64), dict(X=X.float()), dict(X=X.t()), dict(X=X.half()), dict(Wf_values=v[:-1]), dict(Wf_values=v.float()), dict(Wf_index=idx[:-1]), dict(bias=R[0].float()), dict(bias=R[0, :60]),
                dict(residual=R.float()), dict(residual=R[:5]), dict(residual=R.t()), dict(Y=X), dict(ckpt=R), dict(ckpt=torch.zeros((6, 66, 2), dtype=torch.uint8, device="cuda")[:, :, 0])):
        with pytest.raises((ValueError, TypeError)):
            f(**bad)
    for bad, status in ((dict(act=7), 5), (dict(ckpt=torch.zeros((65,), dtype=torch.uint8, device="cuda")), 6), (dict(I=62, Wf_values=v), 2), (dict(residual=R, Y=torch.as_strided(R, (6, 64), (64, 1), 0)[:6]), 0)):
        if status == 0:
            f(**bad)                                                   # the same memory under another name: in place
            continue
        with pytest.raises(bm.BimaskError) as e:
            f(**bad)
        assert e.value.status == status
    ck = bm.bimask_checkpoint_store(X)
    for call in (lambda: bm.bimask_checkpoint_store(X[0]), lambda: bm.bimask_checkpoint_store(X.half()), lambda: bm.bimask_checkpoint_load(ck.view(torch.int32), 6, 128), lambda: bm.bimask_checkpoint_load(ck, 6, 128, X=R),
                 lambda: bm.bimask_act_bwd(R, ck, 1, dZ=X), lambda: bm.bimask_act_bwd(R, ck, 1, dbias=R[0]), lambda: bm.bimask_weight_grad(R, ck, 128, dW=R), lambda: bm.bimask_weight_grad(R, ck, 128, accumulate=True),
                 lambda: bm.bimask_weight_grad(R.t(), ck, 128), lambda: bm.bimask_weight_grad(R, ck, 128, dw_dtype=torch.float16)):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call, status in ((lambda: bm.bimask_checkpoint_load(ck, 7, 128), 6), (lambda: bm.bimask_act_bwd(R, None, 2), 1), (lambda: bm.bimask_act_bwd(R, ck, 2, want_dZ=False, want_dbias=False), 1),
                         (lambda: bm.bimask_weight_grad(R, ck, 129), 6), (lambda: bm.bimask_weight_grad(R.float(), ck, 128, dw_dtype=torch.bfloat16), 4), (lambda: bm.bimask_act_bwd(R[:1].expand(6, 64), ck, 0), 2)):
        with pytest.raises(bm.BimaskError) as e:
            call()
        assert e.value.status == status


# ---- activations over their whole range ----------------------------------------------------------------------------------------------
def range_of_z(dtype, n):
    """n pre-activations that the type holds: every magnitude of bf16 from 2^-20 to 2^7, of fp32 as many, the largest ones and zeros."""
    if dtype == BF:
        z = (np.arange((127 - 20) << 7, (127 + 7) << 7, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)
    else:
        rng = np.random.default_rng(37)
        z = rounded(np.concatenate((np.exp2(rng.uniform(-20, 7, 6000)), rng.uniform(0, 15, 6000))), F32)
    z = np.concatenate((z, -z, rounded([0.0, -0.0, 1e20, -1e20, 3e38, -3e38], dtype)))
    return np.resize(z, n)


def half_step(v, dtype):
    """Half the distance of the type's values around v."""
    bits = 7 if dtype == BF else 23
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - bits - 1)


@pytest.mark.parametrize("a", ref.ACTS)
@pytest.mark.parametrize("I,T,N,M,dtype", [(64, 120, 2, 4, BF), (512, 8200, 2, 4, BF), (512, 8200, 4, 8, BF), (64, 400, 2, 4, F32)])
def test_activations_over_their_range(I, T, N, M, dtype, a):
    """Weights that hand every feature through, nothing added: the activation alone, in the epilogues of the streaming, wide and fp32 kernels.
    The accuracy that the header states: (32 + 3 u) 2^-24 relative, results below 2^-119 (where an exponential of fp32 ends) may be 0;
    then one rounding."""
    v, idx = operand(np.eye(I), N, M, dtype)
    z = range_of_z(dtype, T * I).reshape(T, I)
    got = from_dev_f64(bm.bimask_sparse_linear_fwd(dev(z, dtype), v, idx, I, I, N, M, act=bm.ACTS[a])[0], dtype)
    with np.errstate(over="ignore"):                                   # (1 + tanh(u)) / 2 = 1 / (1 + exp(-2u)), which loses no digits to 1 + tanh
        want = z / (1.0 + np.exp(-np.sqrt(8.0 / np.pi) * (z + 0.044715 * z ** 3))) if a == "gelu_tanh" else ref.act(z, a)
    u = {"gelu": z * z / 2, "silu": np.abs(z), "gelu_tanh": 1.6 * np.abs(z) + 0.072 * np.abs(z) ** 3}.get(a, z)
    # (beyond z = 15 the activation is z or below 2^-119)
    off = 0.0 if a in ("none", "relu") else (32 + 3 * np.minimum(u, 120.0)) * 2.0 ** -24 * np.abs(want) + 2.0 ** -119
    bad = np.abs(got - want) > half_step(np.abs(want) + off, dtype) + off
    assert not bad.any(), (bad.sum(), z[bad][:5], got[bad][:5], want[bad][:5])


# ---- ragged large products, blocks of zeros, infinities in checkpoints -----------------------------------------------------------------
# (I, J, T, N, M, type): the streaming forms, split and not, both wide forms, the large form and fp32, the features no whole blocks of 32
FORMS = [(100, 2184, 3, 2, 4, BF), (104, 648, 70, 4, 8, BF), (72, 128, 1000, 2, 4, BF), (520, 384, 8200, 2, 4, BF), (520, 384, 8200, 4, 8, BF), (1032, 1024, 21900, 2, 4, BF), (40, 64, 70, 2, 4, F32)]


def exact_sums(X, W):
    """X W^T of small integers: exact in fp32, whatever the order."""
    return (X.astype(np.float32) @ W.astype(np.float32).T).astype(np.float64)


def test_ragged_large_linear_is_exact():
    """The large product with a last tile of 8 features and 12 tokens: every byte of output and checkpoint, a residual whose rows start on
    4 bytes only, and in place."""
    I, J, T, N, M, _ = FORMS[5]
    rng = np.random.default_rng(41)
    W, Wm = masked_integers(rng, I, J, N, M)
    x, bias, res = few_ones(rng, T, J), rng.integers(-20, 21, I).astype(np.float64), rng.integers(-60, 61, (T, I)).astype(np.float64)
    z = exact_sums(x, Wm) + bias
    codes, scales = ref.store(z)
    v, idx = operand(W, N, M, BF)
    X, b = dev(x, BF), dev(bias[None], BF)[0]
    for pad in (2, 8):                                                 # pitches of 4 and of 16 bytes
        R, _ = strided(res, BF, pad)
        Y, whole = strided(np.full((T, I), 99.0), BF, 8, 0, 99.0)
        _, ck = bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=b, residual=R, Y=Y, want_ckpt=True)
        assert (from_dev_f64(Y, BF) == z + res).all()
        gc, gs = ref.split(ck.cpu().numpy(), T, I)
        assert (gc == codes).all() and (gs == scales).all()
        Y.fill_(99.0)
        assert (whole == 99.0).all(), "written beside or behind the rows"
    bm.bimask_sparse_linear_fwd(X, v, idx, I, J, N, M, bias=b, act=bm.ACT_RELU, residual=R, Y=R)
    assert (from_dev_f64(R, BF) == np.maximum(z, 0.0) + res).all()


@pytest.mark.parametrize("I,J,T,N,M,dtype", FORMS)
def test_blocks_of_zeros_have_the_smallest_scale(I, J, T, N, M, dtype):
    rng = np.random.default_rng(43)
    W, Wm = masked_integers(rng, I, J, N, M)
    x = few_ones(rng, T, J)
    x[1::3] = 0.0
    v, idx = operand(W, N, M, dtype)
    codes, scales = ref.store(exact_sums(x, Wm))
    gc, gs = ref.split(bm.bimask_sparse_linear_fwd(dev(x, dtype), v, idx, I, J, N, M, want_ckpt=True)[1].cpu().numpy(), T, I)
    assert (scales[1] == 1).all() and (gc == codes).all() and (gs == scales).all()
    gc, gs = ref.split(bm.bimask_checkpoint_store(dev(x, dtype)).cpu().numpy(), T, J)
    codes, scales = ref.store(x)
    assert (gc == codes).all() and (gs == scales).all()


@pytest.mark.parametrize("I,J,T,N,M,dtype", FORMS)
def test_infinities_and_nan_reach_their_own_blocks_of_a_checkpoint(I, J, T, N, M, dtype):
    """By token (its sums infinite or NaN) and by feature (an infinite bias): scale byte 255 and codes 0 there, no other byte changes."""
    rng = np.random.default_rng(47)
    W, _ = masked_integers(rng, I, J, N, M)
    v, idx = operand(np.abs(W), N, M, dtype)
    x, bias = few_ones(rng, T, J), np.ones(I)
    call = lambda x, b: bm.bimask_sparse_linear_fwd(dev(x, dtype), v, idx, I, J, N, M, bias=dev(b[None], dtype)[0], act=bm.ACT_RELU, want_ckpt=True)  # noqa: E731
    clean, k0 = call(x, bias)
    c0, s0 = ref.split(k0.cpu().numpy(), T, I)
    bad_x = x.copy()
    bad_x[1], bad_x[T - 1] = 3e38, np.nan                              # sums of like signs beyond bf16 and fp32: +inf
    keep = np.setdiff1d(np.arange(T), [1, T - 1])
    Y, k = call(bad_x, bias)
    c, s = ref.split(k.cpu().numpy(), T, I)
    assert (s[[1, T - 1]] == 255).all() and (c[[1, T - 1]] == 0).all() and (c[keep] == c0[keep]).all() and (s[keep] == s0[keep]).all()
    y, y0 = from_dev_f64(Y, dtype), from_dev_f64(clean, dtype)
    assert np.isposinf(y[1]).all() and np.isnan(y[T - 1]).all() and (y[keep] == y0[keep]).all()
    bias[I - 3] = -np.inf                                              # in the last block, which has features that do not exist
    last = (I - 3) // 32
    Y, k = call(x, bias)
    c, s = ref.split(k.cpu().numpy(), T, I)
    assert (s[:, last] == 255).all() and (c[:, 32 * last:32 * last + 32] == 0).all()
    assert (s[:, :last] == s0[:, :last]).all() and (c[:, :32 * last] == c0[:, :32 * last]).all()
    y = from_dev_f64(Y, dtype)
    assert (y[:, I - 3] == 0).all() and (np.delete(y, I - 3, 1) == np.delete(y0, I - 3, 1)).all()
