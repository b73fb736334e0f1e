"""What the training-step operators refuse, through the C ABI and the binding;
none of it reaches a device (the GPU part passes page-locked host memory, which
is refused before any launch)."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

INVALID, DTYPE, ALIGN, UNSUPPORTED = 1, 2, 3, 6
BASE = 1 << 20        # an address that no check reads


@pytest.fixture(scope="module")
def L():
    from paper_2605_19811_gb300 import build, lionmuon
    build.build()
    lionmuon.load_library()
    return lionmuon


def mat(L, rows=4, cols=8, ld=None, dtype=1, data=BASE):
    return L.LmMatrix(data, rows, cols, cols if ld is None else ld, dtype)


def code(L, rows=4, cols=8, ld=16, lds=4, fmt=0, codes=BASE, scales=BASE):
    return L.LmCheckpoint8(codes, scales, rows, cols, ld, lds, fmt)


def ref(x):
    return None if x is None else ctypes.byref(x)


def logprob(L, fn="lm_token_logprob", **kw):
    a = L.LmTokenLogprobArgs()
    a.logits, a.targets, a.logp, a.entropy, a.lse = mat(L), BASE, BASE, BASE, BASE
    for k, v in kw.items():
        setattr(a, k, v)
    return getattr(L.load_library(), fn)(ctypes.byref(a), None)


def test_struct_sizes_match_the_header(L, tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "lionmuon.h"\nint main(void){printf("%zu %zu %zu", sizeof(lm_matrix), '
                   'sizeof(lm_checkpoint8), sizeof(lm_token_logprob_args));return 0;}')
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(c) for c in (L.LmMatrix, L.LmCheckpoint8, L.LmTokenLogprobArgs)]


def test_logprob_refusals(L):
    lib = L.load_library()
    assert lib.lm_token_logprob(None, None) == INVALID
    assert logprob(L, logits=mat(L, dtype=7)) == DTYPE
    assert logprob(L, logits=mat(L, data=0)) == INVALID
    assert logprob(L, logits=mat(L, data=BASE + 1)) == ALIGN
    assert logprob(L, logits=mat(L, dtype=0, data=BASE + 2)) == ALIGN
    assert logprob(L, logits=mat(L, ld=7)) == INVALID
    assert logprob(L, logits=mat(L, rows=-1)) == INVALID
    assert logprob(L, logits=mat(L, cols=0)) == INVALID
    assert logprob(L, logits=mat(L, cols=1 << 31)) == UNSUPPORTED
    assert logprob(L, logits=mat(L, rows=1 << 20, ld=1 << 50)) == UNSUPPORTED
    assert logprob(L, targets=None) == INVALID
    assert logprob(L, targets=BASE + 4) == ALIGN
    for k in (-1, 9, 33):
        assert logprob(L, top_k=k, top_logp=BASE, top_index=BASE) == INVALID
    assert logprob(L, top_k=2) == INVALID
    assert logprob(L, top_logp=BASE, top_index=BASE) == INVALID
    assert logprob(L, g_logp=BASE) == INVALID                                 # weights without dlogits
    assert logprob(L, dlogits=mat(L)) == INVALID                              # dlogits without weights
    assert logprob(L, dlogits=mat(L, dtype=0), g_logp=BASE) == DTYPE
    assert logprob(L, dlogits=mat(L, cols=9), g_logp=BASE) == INVALID
    assert logprob(L, dlogits=mat(L, ld=16), g_logp=BASE) == INVALID          # over the logits, another pitch
    assert logprob(L, lse=BASE + 2) == ALIGN
    g = "lm_token_logprob_grad"
    assert logprob(L, g, g_logp=BASE) == INVALID
    assert logprob(L, g, g_logp=BASE, dlogits=mat(L), lse=None) == INVALID
    assert logprob(L, g, g_entropy=BASE, dlogits=mat(L), entropy=None) == INVALID
    assert logprob(L, logits=mat(L, rows=0), top_k=0) == 0                    # nothing to do
    assert lib.lm_last_error() != b""


def test_norm_refusals(L):
    lib = L.load_library()

    def fwd(x=mat(L), r=None, w=None, eps=1e-6, h=None, y=None, rstd=None, kept=None):
        return lib.lm_rmsnorm(ref(x), ref(r), ref(w), eps, ref(h), ref(y), rstd, ref(kept), None)

    assert fwd(x=None) == INVALID
    for eps in (-1e-9, float("nan"), float("inf")):
        assert fwd(eps=eps) == INVALID
    assert fwd(h=mat(L)) == INVALID
    assert fwd(r=mat(L, rows=3)) == INVALID
    assert fwd(r=mat(L, dtype=0)) == DTYPE
    assert fwd(y=mat(L, dtype=0)) == DTYPE
    assert fwd(r=mat(L), h=mat(L, ld=16)) == INVALID                          # over x, another pitch
    assert fwd(w=L.LmTensor(BASE, 1, 7, 1)) == INVALID
    assert fwd(w=L.LmTensor(BASE, 1, 8, 3)) == DTYPE
    assert fwd(w=L.LmTensor(BASE + 1, 1, 8, 1)) == ALIGN
    assert fwd(kept=code(L, cols=9)) == INVALID
    assert fwd(kept=code(L, fmt=2)) == DTYPE
    assert fwd(kept=code(L, ld=24)) == ALIGN
    assert fwd(kept=code(L, codes=BASE + 8)) == ALIGN
    assert fwd(kept=code(L, lds=3)) == INVALID
    assert fwd(rstd=BASE + 1) == ALIGN
    assert fwd(x=mat(L, rows=0), r=mat(L, rows=0)) == 0

    v = L.LmTensor(BASE, 1, 8, 0)

    def bwd(dy=mat(L), h=mat(L), h8=None, rstd=BASE, w=None, dh=None, dx=mat(L), dw=None, ws=BASE, n=1 << 20):
        return lib.lm_rmsnorm_grad(ref(dy), ref(h), ref(h8), rstd, ref(w), ref(dh), ref(dx), ref(dw), ws, n, None)

    assert bwd(dy=None) == INVALID
    assert bwd(h=None) == INVALID
    assert bwd(h8=code(L)) == INVALID                                         # both
    assert bwd(dx=None) == INVALID
    assert bwd(rstd=None) == INVALID
    assert bwd(dh=mat(L, dtype=0)) == DTYPE
    assert bwd(dx=mat(L, ld=16)) == INVALID                                   # over dy, another pitch
    assert bwd(dw=v, n=16) == INVALID
    assert bwd(dw=v, ws=None) == INVALID
    assert bwd(dw=v, ws=BASE + 8) == ALIGN
    assert bwd(dw=L.LmTensor(BASE, 2, 4, 0)) == INVALID
    assert lib.lm_rmsnorm_grad_workspace(0, 8) == 0 and lib.lm_rmsnorm_grad_workspace(-1, 8) == 0
    assert lib.lm_rmsnorm_grad_workspace(4, 8) > 0


def test_checkpoint_refusals(L):
    lib = L.load_library()
    for fn in (lambda x, c: lib.lm_checkpoint8_pack(ref(x), ref(c), None), lambda x, c: lib.lm_checkpoint8_unpack(ref(c), ref(x), None)):
        assert fn(None, code(L)) == INVALID and fn(mat(L), None) == INVALID
        assert fn(mat(L, dtype=2), code(L)) == DTYPE
        assert fn(mat(L, cols=7), code(L)) == INVALID
        assert fn(mat(L), code(L, codes=0)) == INVALID
        assert fn(mat(L), code(L, scales=0)) == INVALID
        assert fn(mat(L), code(L, scales=BASE + 2)) == ALIGN
        assert fn(mat(L, rows=0), code(L, rows=0)) == 0

    def wg(dy=mat(L), x=code(L), dw=mat(L, rows=8), acc=0, ws=BASE, n=1 << 30):
        return lib.lm_linear_wgrad8(ref(dy), ref(x), ref(dw), acc, ws, n, None)

    assert wg(dy=None) == INVALID and wg(x=None) == INVALID and wg(dw=None) == INVALID
    assert wg(dy=mat(L, rows=5)) == INVALID
    assert wg(dw=mat(L, rows=7)) == INVALID
    assert wg(dw=mat(L, rows=8, dtype=4)) == DTYPE
    assert wg(dw=mat(L, rows=8, ld=4)) == INVALID
    assert wg(x=code(L, ld=8)) == ALIGN
    n, m = 1 << 30, 1 << 10
    assert wg(dy=mat(L, rows=n, cols=m), x=code(L, rows=n, lds=n), dw=mat(L, rows=m)) == UNSUPPORTED
    assert wg(dy=mat(L, cols=0), dw=mat(L, rows=0)) == 0


def test_binding_refusals(L):
    from paper_2605_19811_gb300 import training as T
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        T._matrix(x.t(), "x")
    with pytest.raises(ValueError):
        T._matrix(torch.zeros(2, 3, 8).transpose(0, 1), "x")
    with pytest.raises(ValueError):
        T._matrix(torch.zeros(4, 1).expand(4, 8), "x")
    with pytest.raises(ValueError):
        T._matrix(torch.tensor(1.0), "x")
    with pytest.raises(TypeError):
        T._matrix(x.half(), "x")
    with pytest.raises(TypeError):
        T._array(torch.zeros(4, dtype=torch.int32), 4, torch.int64, "targets")
    with pytest.raises(ValueError):
        T._array(torch.zeros(5, dtype=torch.int64), 4, torch.int64, "targets")
    m = T._matrix(torch.zeros(2, 3, 8), "x")
    assert (m.rows, m.cols, m.ld) == (6, 8, 8)
    m = T._matrix(torch.zeros(8), "x")
    assert (m.rows, m.cols) == (1, 8)
    codes, scales = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(1, 4)
    with pytest.raises(ValueError):
        T.Checkpoint8(codes, scales, 8, "int8")
    with pytest.raises(ValueError):
        T.Checkpoint8(codes, scales, 17, "i8")
    with pytest.raises(ValueError):
        T.Checkpoint8(codes, torch.zeros(1, 3), 8, "i8")
    with pytest.raises(TypeError):
        T.Checkpoint8(codes.to(torch.int8), scales, 8, "i8")
    with pytest.raises(ValueError):
        T.linear_wgrad8(x, T.Checkpoint8(codes, scales, 8, "i8"), accumulate=True)


@pytest.mark.gpu
def test_host_memory_is_refused(L):
    from paper_2605_19811_gb300 import training as T
    host, dev = torch.zeros(4, 8).pin_memory(), torch.zeros(4, 8, device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    w = torch.ones(8, device="cuda")
    rstd = torch.ones(4, device="cuda")
    ck = T.checkpoint8(dev, "i8")
    host_ck = T.Checkpoint8(ck.codes.cpu().pin_memory(), ck.scales, 8, "i8")
    calls = [lambda: T.token_logprob(host, y), lambda: T.token_logprob(dev, y.cpu().pin_memory()),
             lambda: T.token_logprob(dev, y, g_logp=rstd.cpu().pin_memory()),
             lambda: T.token_logprob_grad(dev, y, rstd, rstd, rstd, dlogits=host),
             lambda: T.rmsnorm(host, w), lambda: T.rmsnorm(dev, w.cpu().pin_memory()), lambda: T.rmsnorm(dev, w, residual=host),
             lambda: T.rmsnorm_grad(dev, host, rstd, w), lambda: T.rmsnorm_grad(dev, host_ck, rstd, w),
             lambda: T.checkpoint8(host, "i8"), lambda: host_ck.unpack(), lambda: T.linear_wgrad8(dev, host_ck),
             lambda: T.linear_wgrad8(host, ck), lambda: T.linear_wgrad8(dev, ck, out=torch.zeros(8, 8).pin_memory())]
    for call in calls:
        with pytest.raises(L.LionMuonError) as e:
            call()
        assert e.value.status == INVALID
    torch.cuda.synchronize()
