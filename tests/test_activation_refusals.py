"""What the activation operators refuse, before anything is launched (no GPU needed), their sizes, and grids for the largest calls
(the library's launches meet tests/launch_recorder.c)."""
import ctypes as C
import os
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2602_08923_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
F, H = B.DQ_F32, B.DQ_BF16
X, Y, Z, W, K, S = (1 << 40) + (0 << 36), (1 << 40) + (1 << 36), (1 << 40) + (2 << 36), (1 << 40) + (3 << 36), (1 << 40) + (4 << 36), (1 << 40) + (5 << 36)
M1, M2, V1, V2 = ((1 << 40) + (i << 36) for i in (6, 7, 8, 9))


def mat(p, dtype=F, ld=64):
    return C.byref(B.Matrix(p, dtype, ld))


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_checkpoint_sizes(L):
    for rows, cols, bytes_ in ((1, 1, 33), (1, 32, 33), (1, 33, 66), (7, 100, 7 * 132), (3, 2048, 3 * 2112), (0, 5, 0), (5, 0, 0), (1 << 40, 1 << 30, 0)):
        assert L.dq_ckpt_bytes(rows, cols) == bytes_ == B.dq_ckpt_bytes(rows, cols)
    assert L.dq_ckpt_bytes(256, 256) == B.dq_mx_packed_bytes(B.DQ_MXFP8_E4M3, 65536)
    assert L.dq_ckpt_bytes(2 ** 63, 2 ** 63) == 0 and L.dq_ckpt_bytes(1, 2 ** 64 - 1) == 0 and L.dq_ckpt_bytes(2 ** 64 - 1, 1) == 0


def test_save_and_load_refuse(L):
    assert L.dq_ckpt_save(None, 4, 64, K, None) == B.DQ_EINVAL
    assert L.dq_ckpt_save(mat(None), 4, 64, K, None) == B.DQ_EINVAL
    assert L.dq_ckpt_save(mat(X), 4, 64, None, None) == B.DQ_EINVAL
    assert L.dq_ckpt_save(mat(X, 2), 4, 64, K, None) == B.DQ_EINVAL
    assert L.dq_ckpt_save(mat(X, F, 63), 4, 64, K, None) == B.DQ_EINVAL          # rows would overlap
    assert L.dq_ckpt_save(mat(X + 2), 4, 64, K, None) == B.DQ_EALIGN
    assert L.dq_ckpt_save(mat(X + 1, H), 4, 64, K, None) == B.DQ_EALIGN
    assert L.dq_ckpt_save(mat(X), 4, 64, K + 8, None) == B.DQ_EALIGN
    assert L.dq_ckpt_save(mat(X), 4, 64, X + 4 * 64 * 4 - 16, None) == B.DQ_EINVAL   # over x's end
    assert L.dq_ckpt_save(mat(X), 4, 64, X - 16, None) == B.DQ_EINVAL
    assert L.dq_ckpt_save(mat(X, F, 1 << 45), 4, 64, K, None) == B.DQ_EUNSUPPORTED
    assert L.dq_ckpt_save(mat(X, F, 1 << 47), 1, 1 << 47, K, None) == B.DQ_EUNSUPPORTED
    assert L.dq_ckpt_load(None, 4, 64, mat(X), None) == B.DQ_EINVAL
    assert L.dq_ckpt_load(K + 1, 4, 64, mat(X), None) == B.DQ_EALIGN
    assert L.dq_ckpt_load(K, 4, 64, mat(K + 16), None) == B.DQ_EINVAL
    assert L.dq_ckpt_load(K, 4, 64, None, None) == B.DQ_EINVAL
    for rows, cols in ((0, 64), (4, 0)):                                        # nothing to do
        assert L.dq_ckpt_save(mat(None), rows, cols, None, None) == B.DQ_OK and L.dq_ckpt_load(None, rows, cols, mat(None), None) == B.DQ_OK


def test_weight_grad_refuses(L):
    def call(dy=mat(X), ck=K, rows=4, outs=64, cols=64, dw=mat(W), db=None, add=0, scratch=S, room=1 << 40):
        return L.dq_ckpt_weight_grad(dy, ck, rows, outs, cols, dw, db, add, scratch, room, None)

    assert call(dy=None) == call(dw=None) == call(ck=None) == call(dy=mat(None)) == call(dw=mat(None)) == B.DQ_EINVAL
    assert call(dy=mat(X, F, 60)) == call(dw=mat(W, F, 60)) == B.DQ_EINVAL
    assert call(ck=K + 4) == call(dw=mat(W + 2)) == call(db=V1 + 2) == call(dw=mat(W, H), db=V1 + 1) == B.DQ_EALIGN
    assert call(dw=mat(X + 64)) == call(dw=mat(K)) == call(db=W + 4) == call(db=X) == B.DQ_EINVAL
    assert call(rows=1 << 31) == call(outs=1 << 31, dy=mat(X, F, 1 << 31)) == call(cols=1 << 31, dw=mat(W, F, 1 << 31)) == B.DQ_EUNSUPPORTED
    assert call(cols=0, db=V1) == B.DQ_EINVAL and call(outs=0) == call(cols=0) == B.DQ_OK
    assert call(rows=0, ck=None, dy=mat(None), add=1) == B.DQ_OK
    rows, outs, cols = 65536, 64, 64                                            # shared out over tokens
    need = L.dq_ckpt_weight_grad_scratch_bytes(H, rows, outs, cols)
    if need:
        big = dict(dy=mat(X, H), rows=rows, outs=outs, cols=cols)
        assert call(**big, scratch=None) == call(**big, room=need - 1) == call(**big, scratch=K) == call(**big, scratch=W) == B.DQ_EINVAL
        assert call(**big, scratch=S + 4) == B.DQ_EALIGN


def test_layer_norm_refuses(L):
    def call(x=mat(X), rows=4, cols=64, w=V1, b=V2, wt=F, eps=1e-5, y=mat(Y), ck=K, mean=M1, rstd=M2):
        return L.dq_layer_norm(x, rows, cols, w, b, wt, eps, y, ck, mean, rstd, None)

    assert call(x=None) == call(y=None) == call(x=mat(None)) == call(y=mat(Y, H)) == call(wt=3) == B.DQ_EINVAL
    assert call(eps=-1e-9) == call(eps=float("nan")) == call(eps=float("inf")) == B.DQ_EINVAL
    assert call(ck=None) == call(mean=None) == call(rstd=None) == call(ck=None, mean=None) == B.DQ_EINVAL
    assert call(ck=K + 8) == call(mean=M1 + 2) == call(rstd=M2 + 1) == call(w=V1 + 2) == call(b=V2 + 1, wt=H) == B.DQ_EALIGN
    assert call(y=mat(X)) == call(y=mat(X + 128)) == call(y=mat(V1)) == call(ck=X) == call(mean=Y) == call(rstd=M1) == call(mean=K) == B.DQ_EINVAL
    assert call(cols=1 << 31, x=mat(X, F, 1 << 31), y=mat(Y, F, 1 << 31)) == B.DQ_EUNSUPPORTED
    assert call(rows=0, x=mat(None), y=mat(None)) == call(cols=0) == B.DQ_OK

    need = L.dq_layer_norm_grad_scratch_bytes(4, 64)
    assert need and L.dq_layer_norm_grad_scratch_bytes(0, 64) == L.dq_layer_norm_grad_scratch_bytes(4, 0) == 0

    def back(dy=mat(X), ck=K, mean=M1, rstd=M2, rows=4, cols=64, w=V1, wt=F, dx=mat(Y), dw=W, db=Z, add=0, scratch=S, room=need):
        return L.dq_layer_norm_grad(dy, ck, mean, rstd, rows, cols, w, wt, dx, dw, db, add, scratch, room, None)

    assert back(dy=None) == back(dx=None) == back(ck=None) == back(mean=None) == back(rstd=None) == back(dx=mat(Y, H)) == back(wt=2) == B.DQ_EINVAL
    assert back(dw=None) == back(db=None) == back(scratch=None) == back(room=need - 1) == B.DQ_EINVAL
    assert back(ck=K + 2) == back(mean=M1 + 1) == back(w=V1 + 2) == back(dw=W + 2) == back(scratch=S + 8) == B.DQ_EALIGN
    assert back(dx=mat(X)) == back(dw=V1) == back(db=W) == back(dw=M1) == back(scratch=X) == back(scratch=W) == back(dx=mat(K)) == B.DQ_EINVAL
    assert back(rows=0, dw=W, db=W) == B.DQ_EINVAL and back(rows=0, dw=W + 1) == B.DQ_EALIGN
    assert back(rows=0, add=1) == back(cols=0) == B.DQ_OK


def test_gate_refuses(L):
    def call(kind=0, z=mat(X), u=mat(Y), rows=4, cols=64, h=mat(Z), cz=K, cu=S):
        return L.dq_gate(kind, z, u, rows, cols, h, cz, cu, None)

    assert call(kind=2) == call(z=None) == call(h=None) == call(u=mat(Y, H)) == call(h=mat(Z, H)) == call(z=mat(None)) == B.DQ_EINVAL
    assert call(cz=None) == call(cu=None) == call(u=None) == call(u=None, cz=None) == B.DQ_EINVAL
    assert call(cz=K + 4) == call(cu=S + 4) == call(u=mat(Y + 2)) == B.DQ_EALIGN
    assert call(h=mat(X)) == call(h=mat(Y + 256)) == call(cz=S) == call(cu=Z) == B.DQ_EINVAL
    # in one wider matrix: z and u side by side are read only; h over the second half of z is refused
    assert call(z=mat(X, F, 128), h=mat(X + 4 * 32, F, 128)) == B.DQ_EINVAL
    assert call(rows=0) == call(cols=0) == B.DQ_OK

    def back(kind=0, dh=mat(X), cz=K, cu=S, rows=4, cols=64, dz=mat(Y, F, 128), du=mat(Y + 4 * 64, F, 128)):
        return L.dq_gate_grad(kind, dh, cz, cu, rows, cols, dz, du, None)

    assert back(kind=-1) == back(dh=None) == back(dz=None) == back(cz=None) == back(cu=None) == back(du=None) == back(dz=mat(Y, H, 128)) == B.DQ_EINVAL
    assert back(cz=K + 1) == back(cu=S + 8) == back(du=mat(Y + 4 * 64 + 1, F, 128)) == B.DQ_EALIGN
    assert back(du=mat(Y + 4 * 63, F, 128)) == back(du=mat(Y, F, 128)) == back(du=mat(Y + 4 * 64, F, 129)) == back(dz=mat(X)) == back(dz=mat(K)) == B.DQ_EINVAL
    assert back(rows=0) == back(cols=0) == B.DQ_OK


@pytest.mark.parametrize("call", [
    lambda x: B.dq_ckpt_save(x),
    lambda x: B.dq_ckpt_load(B.Checkpoint(torch.zeros(66, dtype=torch.uint8), 2, 32)),
    lambda x: B.dq_ckpt_weight_grad(x, B.Checkpoint(torch.zeros(66, dtype=torch.uint8), 2, 32)),
    lambda x: B.dq_layer_norm(x),
    lambda x: B.dq_layer_norm_grad(x, B.SavedNorm(B.Checkpoint(torch.zeros(66, dtype=torch.uint8), 2, 32), torch.zeros(2), torch.zeros(2))),
    lambda x: B.dq_gate(x),
    lambda x: B.dq_gate_grad(x, B.SavedGate("silu", B.Checkpoint(torch.zeros(66, dtype=torch.uint8), 2, 32), None)),
])
def test_tensors_off_the_gpu_are_refused(call):
    with pytest.raises(B.DqError, match="CUDA tensor"):
        call(torch.zeros(2, 32))


def test_kinds_and_saved_sizes():
    with pytest.raises(B.DqError, match="silu and gelu"):
        B.dq_gate(torch.zeros(2, 32), kind="relu")
    d = torch.zeros(66, dtype=torch.uint8)
    with pytest.raises(B.DqError, match="one size"):
        B.dq_gate_grad(torch.zeros(2, 32), B.SavedGate("silu", B.Checkpoint(d, 2, 32), B.Checkpoint(d, 1, 64)))


# ------------------------------------------------------------------------------------ grids
@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("recorder") / "launch_recorder.so")
    subprocess.check_call(["gcc", "-O1", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "launch_recorder.c"), "-o", so])
    return so


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 40), (16384, 2048), (1, 2 ** 31 - 1), (2 ** 31 - 1, 33), (2 ** 20 + 3, 70001)])
def test_every_call_keeps_to_what_hip_launches(recorder, rows, cols):
    body = f"""
        import ctypes as C, sys
        sys.path.insert(0, {os.path.dirname(HERE)!r})
        R = C.CDLL({recorder!r}, mode=C.RTLD_GLOBAL)
        from paper_2602_08923_amd import binding as B
        L = C.CDLL(B.LIB_PATH)
        class Launch(C.Structure):
            _fields_ = [("grid", C.c_uint32 * 3), ("block", C.c_uint32 * 3), ("args", C.c_uint64 * 8)]
        P, U, I, M = C.c_void_p, C.c_uint64, C.c_int, C.POINTER(B.Matrix)
        L.dq_ckpt_save.argtypes = [M, U, U, P, P]
        L.dq_ckpt_load.argtypes = [P, U, U, M, P]
        L.dq_ckpt_weight_grad_scratch_bytes.argtypes, L.dq_ckpt_weight_grad_scratch_bytes.restype = [I, U, U, U], C.c_size_t
        L.dq_ckpt_weight_grad.argtypes = [M, P, U, U, U, M, P, I, P, C.c_size_t, P]
        L.dq_layer_norm.argtypes = [M, U, U, P, P, I, C.c_float, M, P, P, P, P]
        L.dq_layer_norm_grad_scratch_bytes.argtypes, L.dq_layer_norm_grad_scratch_bytes.restype = [U, U], C.c_size_t
        L.dq_layer_norm_grad.argtypes = [M, P, P, P, U, U, P, I, M, P, P, I, P, C.c_size_t, P]
        L.dq_gate.argtypes = [I, M, M, U, U, M, P, P, P]
        L.dq_gate_grad.argtypes = [I, M, P, P, U, U, M, M, P]
        rows, cols = {rows}, {cols}
        at = [1 << 50, 2 << 50, 3 << 50, 4 << 50, 5 << 50, 6 << 50, 7 << 50, 8 << 50, 9 << 50]
        for t in (0, 1):
            m = [B.Matrix(p, t, cols) for p in at]
            assert L.dq_ckpt_save(m[0], rows, cols, at[1], None) == 0
            assert L.dq_ckpt_load(at[1], rows, cols, m[0], None) == 0
            assert L.dq_gate(t, m[0], m[1], rows, cols, m[2], at[3], at[4], None) == 0
            assert L.dq_gate_grad(t, m[0], at[3], at[4], rows, cols, m[1], m[2], None) == 0
            assert L.dq_layer_norm(m[0], rows, cols, at[1], at[2], 0, 1e-5, m[3], at[4], at[5], at[6], None) == 0
            need = L.dq_layer_norm_grad_scratch_bytes(rows, cols)
            assert L.dq_layer_norm_grad(m[0], at[1], at[2], at[3], rows, cols, at[4], t, m[5], at[6], at[7], 0, at[8], need, None) == 0
            for outs in (1, 96, 4099):
                if outs * cols < 1 << 40:
                    g, w = B.Matrix(at[0], t, outs), B.Matrix(at[2], t, cols)
                    need = L.dq_ckpt_weight_grad_scratch_bytes(t, rows, outs, cols)
                    assert need < 1 << 40
                    got = L.dq_ckpt_weight_grad(g, at[1], rows, outs, cols, w, at[3], 0, at[4], need, None)
                    assert got == 0, (outs, got)
        a = (Launch * 4096)()
        n = R.recorded(a, 4096)
        assert n >= 12
        for l in a[:n]:
            assert all(x >= 1 for x in l.grid) and l.grid[1] <= 65535 and l.grid[2] <= 65535 and all(x * y < 2 ** 32 for x, y in zip(l.grid, l.block))
    """
    got = subprocess.run([sys.executable, "-c", textwrap.dedent(body)], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got.stderr
