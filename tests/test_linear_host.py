"""Host-side checks of the linear layer's calls that need no GPU: sizes, refusals before any launch, and which kernels the GPU tests'
sizes reach (test_dispatch.py's recording library)."""
import ctypes

import pytest

import paper_2302_06058_amd as bm
import test_gpu_linear as gpu
from paper_2302_06058_amd import synth
from test_dispatch import A, B, C, D, E, rec  # noqa: F401

P = ctypes.c_void_p
BIG = 1 << 40
CODE = {synth.BF16: bm.BF16, synth.F32: bm.F32}


def test_checkpoint_sizes():
    assert bm.checkpoint_bytes(1, 1) == 33 and bm.checkpoint_bytes(3, 33) == 3 * 66 and bm.checkpoint_bytes(8192, 11008) == 8192 * 344 * 33
    assert bm.checkpoint_bytes(0, 5) == bm.checkpoint_bytes(5, 0) == bm.checkpoint_bytes(-1, 5) == bm.checkpoint_bytes(1 << 39, 1) == 0


def test_workspaces():
    ws = bm.workspace_bytes
    assert ws(bm.WS_ACT_BWD, 64, 0, 16, 0, bm.BF16, 0, 0) == 0                     # one strip writes the bias gradient itself
    n = ws(bm.WS_ACT_BWD, 1000, 0, 6347, 0, bm.BF16, 0, 0)
    assert n > 0 and n % (1024 * 4) == 0
    assert ws(bm.WS_ACT_BWD, 0, 0, 6347, 0, bm.BF16, 0, 0) == ws(bm.WS_ACT_BWD, 1000, 0, 0, 0, bm.BF16, 0, 0) == 0
    assert ws(bm.WS_WEIGHT_GRAD, 11008, 4096, 8192, 0, bm.BF16, 0, 0) == 0
    n = ws(bm.WS_WEIGHT_GRAD, 64, 576, 200704, 0, bm.BF16, 0, 0)
    assert n > 0 and n % (64 * 576 * 4) == 0
    assert ws(bm.WS_WEIGHT_GRAD, 64, 576, 200704, 0, 9, 0, 0) == 0


def lin(rec_or_lib, X=A, T=32, ldx=128, v=B, idx=C, I=64, J=128, dtype=bm.BF16, N=2, M=4, bias=None, act=0, R=None, ldr=0, Y=D, ldy=64, ck=None, ckb=BIG):
    return rec_or_lib("bimask_sparse_linear_fwd", X, T, ldx, v, idx, I, J, dtype, N, M, bias, act, R, ldr, Y, ldy, ck, ckb, None)


def raw(name, *args):
    return getattr(bm.lib(), name)(*args)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), 1), (dict(v=None), 1), (dict(idx=None), 1), (dict(Y=None), 1), (dict(T=0), 2), (dict(ldx=126), 2), (dict(ldy=60), 2), (dict(I=62), 2), (dict(M=5), 3), (dict(dtype=7), 4),
    (dict(act=-1), 5), (dict(act=5), 5), (dict(bias=E + 8), 7), (dict(R=E, ldr=60), 2), (dict(R=E, ldr=65), 7), (dict(R=E + 2, ldr=64), 7), (dict(ck=E, ckb=32 * 66 - 1), 6), (dict(ck=E + 8), 7),
    (dict(ldx=129), 7), (dict(X=A + 2), 7), (dict(v=B + 8), 7), (dict(idx=C + 4), 7), (dict(T=1 << 39, ldx=128), 2), (dict(T=1 << 38, ldx=1 << 40), 2),
    (dict(Y=A, ldy=128), 5), (dict(Y=A + 32 * 256 - 4), 5),                         # the output on the input
    (dict(R=D, ldr=66), 5), (dict(R=D + 4, ldr=64), 5), (dict(R=D + 31 * 128, ldr=64), 5),      # partly on the residual, or with another pitch
    (dict(ck=D), 5), (dict(ck=A), 5), (dict(ck=E, R=E + 16, ldr=64), 5)])
def test_linear_refusals(kw, want):
    assert lin(raw, **kw) == want


@pytest.mark.parametrize("kw", [
    dict(Y=B), dict(Y=B + 32 * 128 * 2 - 4), dict(Y=C + 4), dict(Y=C - 16 * 128), dict(bias=E, Y=E + 124), dict(bias=D + 32), dict(ck=B), dict(ck=C), dict(bias=E, ck=E - 32 * 66 + 16)])
def test_linear_refuses_outputs_on_operands(kw):
    assert lin(raw, **kw) == 5


def test_linear_takes_what_it_documents(rec):  # noqa: F811
    for kw in (dict(), dict(bias=E), dict(R=E, ldr=64), dict(R=D, ldr=64), dict(R=E + 4, ldr=66), dict(ck=E, ckb=32 * 66), dict(R=D + 32 * 128, ldr=64), dict(idx=None, N=4, M=8),
               dict(Y=A + 2 * 128, ldx=192, ldy=192)):                             # (columns beside X in one buffer)
        st, l = lin(rec, **kw)
        assert st == 0 and len(l) == 1, kw


@pytest.mark.parametrize("args,want", [
    ((None, 4, 64, 64, 1, B, BIG), 1), ((A, 4, 64, 64, 1, None, BIG), 1), ((A, 0, 64, 64, 1, B, BIG), 2), ((A, 4, 0, 64, 1, B, BIG), 2), ((A, 4, 64, 63, 1, B, BIG), 2), ((A, 4, 64, 64, 2, B, BIG), 4),
    ((A + 1, 4, 64, 64, 1, B, BIG), 7), ((A + 2, 4, 64, 64, 0, B, BIG), 7), ((A, 4, 64, 64, 1, B + 8, BIG), 7), ((A, 4, 64, 64, 1, B, 4 * 66 - 1), 6), ((A, 4, 64, 64, 1, A + 496, BIG), 5)])
def test_checkpoint_refusals(args, want):
    X, T, Cc, ld, dt, ck, n = args
    assert raw("bimask_checkpoint_store", X, T, Cc, ld, dt, ck, n, None) == want
    assert raw("bimask_checkpoint_load", ck, n, T, Cc, dt, X, ld, None) == want


def act_bwd(f, dY=A, T=4000, lddy=64, ck=B, ckb=BIG, I=64, dtype=bm.BF16, act=2, dZ=C, lddz=64, db=D, ws=E, wsb=BIG):
    return f("bimask_act_bwd", dY, T, lddy, ck, ckb, I, dtype, act, dZ, lddz, db, ws, wsb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dY=None), 1), (dict(ck=None), 1), (dict(dZ=None, db=None), 1), (dict(T=0), 2), (dict(lddy=63), 2), (dict(lddz=63), 2), (dict(dtype=3), 4), (dict(act=9), 5), (dict(ckb=100), 6), (dict(ws=None), 6),
    (dict(wsb=16), 6), (dict(ws=E + 4), 7), (dict(db=D + 2), 7), (dict(ck=B + 4), 7), (dict(dZ=A + 2), 5), (dict(dZ=A, lddz=66), 5), (dict(dZ=B), 5), (dict(dY=A + 1), 7)])
def test_act_bwd_refusals(kw, want):
    assert act_bwd(raw, **kw) == want


@pytest.mark.parametrize("db", [A, A + 4000 * 128 - 4, B + 32, B + 4000 * 66 - 8, C + 256, C - 252])
def test_act_bwd_refuses_a_bias_gradient_on_its_operands(db):
    assert act_bwd(raw, db=db) == 5


def test_act_bwd_launches(rec):  # noqa: F811
    assert [l.kernel for l in act_bwd(rec)[1]] == ["k_act_bwd", "k_sum_strips"]
    assert [l.kernel for l in act_bwd(rec, T=30, ws=None, wsb=0)[1]] == ["k_act_bwd"]              # a single strip
    assert [l.kernel for l in act_bwd(rec, db=None, ws=None, wsb=0)[1]] == ["k_act_bwd"]
    assert [l.kernel for l in act_bwd(rec, dZ=A)[1]] == ["k_act_bwd", "k_sum_strips"]              # in place
    assert act_bwd(rec, ck=None, act=0, dZ=None)[0] == 0


def grad(f, dY=A, T=4000, lddy=64, ck=B, ckb=BIG, I=64, J=96, dtype=bm.BF16, dW=C, lddw=96, dwt=bm.F32, acc=0, ws=E, wsb=BIG):
    return f("bimask_weight_grad", dY, T, lddy, ck, ckb, I, J, dtype, dW, lddw, dwt, acc, ws, wsb, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dY=None), 1), (dict(ck=None), 1), (dict(dW=None), 1), (dict(T=0), 2), (dict(J=0), 2), (dict(lddw=95), 2), (dict(lddy=63), 2), (dict(dtype=2), 4), (dict(dwt=2), 4),
    (dict(dtype=bm.F32, dwt=bm.BF16), 4), (dict(acc=2), 5), (dict(ckb=4000 * 99 - 1), 6), (dict(ws=None), 6), (dict(wsb=64), 6), (dict(ws=E + 8), 7), (dict(ck=B + 1), 7), (dict(dW=C + 2), 7), (dict(dW=A), 5),
    (dict(dW=B + 4000), 5)])
def test_weight_grad_refusals(kw, want):
    assert grad(raw, **kw) == want


@pytest.mark.parametrize("I,J,first", [(4360, 4090, 4096), (4100, 4096, 3840), (5120, 5120, 0), (4096, 4096, 0), (11008, 4096, 0), (4352, 4096, 4096)])
def test_rows_behind_the_whole_rounds_of_a_weight_gradient(rec, I, J, first):  # noqa: F811
    """Two launches that cover dW once, and the second's sums where it splits the tokens; its workspace is what the call asks for."""
    need = bm.workspace_bytes(bm.WS_WEIGHT_GRAD, I, J, 770, 0, bm.BF16, 0, 0)
    assert need == (bm.workspace_bytes(bm.WS_WEIGHT_GRAD, I - first, J, 770, 0, bm.BF16, 0, 0) if first else need)
    st, l = grad(rec, T=770, I=I, J=J, lddy=I, lddw=J, wsb=need)
    assert st == 0
    if first:
        assert len(l) == (3 if need else 2) and l[0].kernel == "k_weight_grad" and l[1].kernel == "k_weight_grad"
    else:
        assert len([x for x in l if x.kernel == "k_weight_grad"]) == 1
    if need:
        assert grad(rec, T=770, I=I, J=J, lddy=I, lddw=J, wsb=need - 1)[0] == 6


def test_wrappers_refuse_tensors_that_are_not_on_the_gpu():
    import torch
    x, b = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4 * 66,), dtype=torch.uint8)
    for call in (lambda: bm.bimask_checkpoint_store(x), lambda: bm.bimask_checkpoint_load(b, 4, 64), lambda: bm.bimask_sparse_linear_fwd(x, x, x, 64, 64, 2, 4),
                 lambda: bm.bimask_act_bwd(x, b, bm.ACT_RELU), lambda: bm.bimask_weight_grad(x, b, 64)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_grids_stay_within_a_launch(rec):  # noqa: F811
    for dt in (bm.BF16, bm.F32):                                       # (the fixture checks the dimensions)
        for T, Cc in ((1 << 33, 8), (1, 0x7FFFFFFF), (1 << 20, 1 << 15)):
            assert rec("bimask_checkpoint_store", A, T, Cc, Cc, dt, B << 20, 1 << 60, None)[0] == 0
            assert rec("bimask_checkpoint_load", B << 20, 1 << 60, T, Cc, dt, A, Cc, None)[0] == 0
            assert act_bwd(rec, T=T, I=Cc, lddy=Cc, lddz=Cc, dtype=dt, ck=B << 20, ckb=1 << 60, dZ=C << 20, db=D << 20, wsb=1 << 60)[0] == 0
        for I, J, T in ((1 << 16, 8, 1 << 22), (8, 1 << 20, 100), (4, 4, 1 << 31)):
            assert lin(rec, I=I, J=J, T=T, ldx=J, ldy=I, dtype=dt, Y=D << 20)[0] in (0, 2)
            assert grad(rec, I=I, J=J, T=T, lddy=I, lddw=J, dtype=dt, ck=B << 20, ckb=1 << 60, dW=C << 20, wsb=1 << 60)[0] == 0


def test_gpu_tests_reach_every_instance_of_the_kernels(rec):  # noqa: F811
    reached = set()
    for I, J, T, N, M, dt, pad in gpu.LINEAR:
        st, l = lin(rec, I=I, J=J, T=T, ldx=J + pad, N=N, M=M, dtype=CODE[dt], Y=D, ldy=I + pad)
        assert st == 0
        reached.update(l)
    for I, J, T, N, M in gpu.LARGE:
        reached.update(lin(rec, I=I, J=J, T=T, ldx=J, N=N, M=M, ldy=I)[1])
    for T, Cc in gpu.CKPT_SHAPES:
        for dt in (bm.BF16, bm.F32):
            reached.update(rec("bimask_checkpoint_store", A, T, Cc, Cc, dt, B, BIG, None)[1])
            reached.update(rec("bimask_checkpoint_load", B, BIG, T, Cc, dt, A, Cc, None)[1])
    for T, I in gpu.ACT_SHAPES:
        for dt in (bm.BF16, bm.F32):
            reached.update(act_bwd(rec, T=T, I=I, lddy=I, lddz=I, dtype=dt)[1])
    for I, J, T, dt, dw, pad in gpu.GRADS:
        st, l = grad(rec, I=I, J=J, T=T, lddy=I + pad, dtype=CODE[dt], dwt=CODE[dw], lddw=J + pad)
        assert st == 0
        reached.update(l)
    names = {f"{l.kernel}<{l.args}>" if l.args else l.kernel for l in reached}
    families = ("k_linear", "k_checkpoint", "k_act_bwd", "k_sum_strips", "k_sum_pieces", "k_sum_few_pieces", "k_weight_grad")
    missing = {k for k in rec.lib.stub_kernels().decode().splitlines() if k.startswith(families)} - names
    assert not missing, sorted(missing)


def test_tensors_of_another_device_are_refused(monkeypatch):
    class Tensor:
        is_cuda = True

        def get_device(self):
            return 1

    monkeypatch.setattr(bm, "_device_index", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        bm._on_current_device(None, Tensor())
    monkeypatch.setattr(bm, "_device_index", lambda: 1)
    bm._on_current_device(Tensor(), None)


@pytest.mark.parametrize("T,J", [(1 << 38, 0x7FFFFFFF), (1 << 38, 1 << 30), (1 << 30, 1 << 28)])
def test_checkpoints_too_large_to_count_are_refused(rec, T, J):  # noqa: F811
    assert bm.checkpoint_bytes(T, J) == 0
    assert grad(rec, T=T, I=4, J=J, lddy=4, lddw=J, ckb=16, wsb=1 << 62)[0] == 2
    assert rec("bimask_checkpoint_load", B, 16, T, J, bm.F32, A, J, None)[0] == 2


def test_weight_gradients_count_their_stages(rec):  # noqa: F811
    """A workgroup counts its stages of 32 tokens in 31 bits: more than 2^30 of them are refused (no card holds such operands)."""
    for T, want in ((1 << 35, 0), ((1 << 35) + 1, 2), (1 << 36, 2), (1 << 38, 2)):
        assert grad(rec, dY=1 << 44, T=T, I=4, J=128 * 256, lddy=4, lddw=128 * 256, ck=1 << 54, ckb=1 << 62, dW=1 << 60, wsb=1 << 62)[0] == want


@pytest.fixture
def on_host(monkeypatch):
    """Wrappers on host tensors, taken for those of the current device; every call of the library is recorded, none is made."""
    import torch
    calls = []

    class Recorder:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)
            return lambda *args: calls.append(name) or 0

    real = bm.lib()
    monkeypatch.setattr(bm, "_torch", torch)
    monkeypatch.setattr(bm, "_device_index", lambda: -1)
    monkeypatch.setattr(bm, "_raw_stream", lambda _: 0)
    monkeypatch.setattr(bm, "lib", lambda: Recorder())
    return calls


def test_wrappers_refuse_operands_that_are_not_contiguous(on_host):
    import torch
    x = torch.zeros((6, 128), dtype=torch.bfloat16)
    v, idx = torch.zeros((64 * 64,), dtype=torch.bfloat16), torch.zeros((64 * 4,), dtype=torch.int32)
    bm.bimask_sparse_linear_fwd(x, v, idx, 64, 128, 2, 4)
    bm.bimask_sparse_linear_fwd(x, v.view(32, -1), idx.view(torch.uint32).view(2, -1), 64, 128, 2, 4)
    bm.bimask_sparse_linear_fwd(x, torch.zeros((64 * 128,), dtype=torch.bfloat16), None, 64, 128, 4, 8)
    assert on_host == ["bimask_sparse_linear_fwd"] * 3
    del on_host[:]
    for values, index, N, M in ((v[:1].expand(64 * 64), idx, 2, 4), (torch.zeros((64 * 64, 2), dtype=torch.bfloat16)[:, 0], idx, 2, 4), (v, idx[:1].expand(64 * 4), 2, 4),
                                (v, torch.zeros((64 * 4, 2), dtype=torch.int32)[:, 1], 2, 4), (v, idx.to(torch.int16), 2, 4), (v, idx.float(), 2, 4), (v, idx.to(torch.uint8), 2, 4), (v, idx.long(), 2, 4),
                                (v[:1].expand(64 * 128), None, 4, 8)):
        with pytest.raises(ValueError):
            bm.bimask_sparse_linear_fwd(x, values, index, 64, 128, N, M)
    assert not on_host


def test_wrappers_refuse_workspaces_that_are_not_contiguous(on_host):
    import torch
    dY, ck = torch.zeros((4000, 64), dtype=torch.bfloat16), torch.zeros((4000 * 99,), dtype=torch.uint8)
    for kind, call in ((bm.WS_ACT_BWD, lambda ws: bm.bimask_act_bwd(dY, None, bm.ACT_NONE, workspace=ws)), (bm.WS_WEIGHT_GRAD, lambda ws: bm.bimask_weight_grad(dY, ck, 96, workspace=ws))):
        need = bm.workspace_bytes(kind, 64, 96, 4000, 0, bm.BF16, 0, 0)
        assert need > 0
        call(torch.zeros((need,), dtype=torch.uint8))
        call(torch.zeros((need // 4,), dtype=torch.float32))
        assert len(on_host) == 2
        del on_host[:]
        for ws in (torch.zeros((1,), dtype=torch.uint8).expand(need), torch.zeros((need, 2), dtype=torch.uint8)[:, 0], torch.zeros((2, need), dtype=torch.uint8)[:, ::2]):
            with pytest.raises(ValueError):
                call(ws)
        assert not on_host
