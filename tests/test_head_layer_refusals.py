"""What the head's, the 8-bit layer's and the queries' and keys' operators
refuse, through the C ABI and the binding; none of it reaches a device."""

import ctypes
import os
import shutil
import subprocess

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


def code(L, rows=4, cols=8, ld=16, lds=4, fmt=1, codes=BASE, scales=BASE):
    return L.LmCheckpoint8(codes, scales, rows, cols, ld, lds, fmt)


def weight(L, rows=6, cols=8, ld=16, lds=1, codes=BASE, scales=BASE):
    return L.LmWeight8(codes, scales, rows, cols, ld, lds)


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_struct_sizes_match_the_header(L, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    names = ("lm_linear_logprob_args", "lm_weight8", "lm_heads", "lm_rotary_part", "lm_qk_rotary_args")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "lionmuon.h"\nint main(void){' + "".join(f'printf("%zu ", sizeof({n}));' for n in names) + "return 0;}")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(c) for c in (L.LmLinearLogprobArgs, L.LmWeight8, L.LmHeads, L.LmRotaryPart, L.LmQkRotaryArgs)]


def test_linear_logprob_refusals(L):
    lib = L.load_library()

    def call(fn="lm_linear_logprob", ws=BASE, n=1 << 40, **kw):
        a = L.LmLinearLogprobArgs()
        a.h, a.weight, a.targets, a.logp, a.entropy, a.lse = mat(L), mat(L, rows=10), BASE, BASE, BASE, BASE
        for k, v in kw.items():
            setattr(a, k, v)
        return getattr(lib, fn)(ctypes.byref(a), ws, n, None)

    g = dict(g_logp=BASE, dh=mat(L))
    assert lib.lm_linear_logprob(None, None, 0, None) == INVALID and lib.lm_linear_logprob_workspace(None) == 0
    assert call(h=mat(L, dtype=0)) == DTYPE and call(weight=mat(L, rows=10, dtype=0)) == DTYPE and call(h=mat(L, dtype=2)) == DTYPE
    assert call(weight=mat(L, rows=10, cols=9)) == INVALID
    assert call(weight=mat(L, rows=0)) == INVALID and call(h=mat(L, cols=0), weight=mat(L, rows=10, cols=0)) == INVALID
    assert call(h=mat(L, data=0)) == INVALID and call(h=mat(L, data=BASE + 1)) == ALIGN and call(h=mat(L, ld=7)) == INVALID
    assert call(h=mat(L, rows=-1)) == INVALID and call(h=mat(L, rows=1 << 32)) == UNSUPPORTED
    assert call(h=mat(L, rows=1 << 30), weight=mat(L, rows=1 << 20)) == UNSUPPORTED
    assert call(h=mat(L, rows=1 << 27)) == UNSUPPORTED
    assert call(h=mat(L, ld=1 << 37)) == UNSUPPORTED
    assert call(targets=None) == INVALID and call(targets=BASE + 4) == ALIGN and call(lse=BASE + 2) == ALIGN
    assert call(dh=mat(L)) == INVALID and call(g_logp=BASE) == INVALID and call(g_lse=BASE) == INVALID
    assert call(**{**g, "dh": mat(L, dtype=0)}) == DTYPE and call(**{**g, "dh": mat(L, rows=5)}) == INVALID
    assert call(g_lse=BASE, dweight=mat(L, rows=9)) == INVALID and call(g_lse=BASE, dweight=mat(L, rows=10, dtype=3)) == DTYPE
    assert call(n=16) == INVALID and call(ws=None) == INVALID and call(ws=BASE + 128) == ALIGN
    f = "lm_linear_logprob_grad"
    assert call(f, g_logp=BASE) == INVALID and call(f, dh=mat(L)) == INVALID
    assert call(f, **g, lse=None) == INVALID and call(f, dh=mat(L), g_entropy=BASE, entropy=None) == INVALID
    assert call(f, **g, targets=None) == INVALID
    assert call(h=mat(L, rows=0)) == 0 and call(f, h=mat(L, rows=0), g_logp=BASE, dh=mat(L, rows=0)) == 0
    assert call(h=mat(L, rows=0), g_lse=BASE, dweight=mat(L, rows=10), accumulate=1) == 0


def test_linear_logprob_workspace_is_bounded(L):
    """16-bit logits of a piece of the tokens take at most 512 MB, or 1024 rows
    of them; 12 bytes of statistics for each half tile of a strip and 4 for each
    half tile, 28 bytes a row, fp32 sums of dW and 40 MB beside them."""
    lib = L.load_library()

    def need(rows, width, vocab, grad):
        a = L.LmLinearLogprobArgs()
        a.h, a.weight = mat(L, rows, width), mat(L, vocab, width)
        if grad:
            a.g_lse, a.dh, a.dweight = BASE, mat(L, rows, width), mat(L, vocab, width)
        return lib.lm_linear_logprob_workspace(ctypes.byref(a))

    assert 0 < need(1, 768, 50304, False) < 1 << 20
    assert need(16384, 768, 50304, False) < 1 << 28
    for rows, width, vocab in ((16384, 768, 50304), (4096, 4096, 50257), (1 << 20, 64, 160000), (7, 64, 1 << 20)):
        most = max(1 << 29, 1024 * vocab * 2)
        assert need(rows, width, vocab, True) <= most * (1 + (12 + 4) / 256 + 0.01) + 4 * vocab * width + (42 << 20)


def test_weight8_refusals(L):
    lib = L.load_library()
    for fn in (lambda w, c: lib.lm_weight8_pack(ref(w), ref(c), None), lambda w, c: lib.lm_weight8_unpack(ref(c), ref(w), None)):
        w = mat(L, rows=6)
        assert fn(None, weight(L)) == INVALID and fn(w, None) == INVALID
        assert fn(mat(L, rows=6, dtype=2), weight(L)) == DTYPE
        assert fn(mat(L, rows=6, cols=7), weight(L)) == INVALID and fn(mat(L, rows=5), weight(L)) == INVALID
        assert fn(w, weight(L, codes=0)) == INVALID and fn(w, weight(L, scales=0)) == INVALID
        assert fn(w, weight(L, scales=BASE + 2)) == ALIGN and fn(w, weight(L, codes=BASE + 8)) == ALIGN and fn(w, weight(L, ld=24)) == ALIGN
        assert fn(mat(L, rows=6, cols=200), weight(L, cols=200, ld=208)) == INVALID                  # two blocks across, pitch 1
        assert fn(mat(L, rows=0), weight(L, rows=0)) == 0


def test_linear8_refusals(L):
    lib = L.load_library()

    def call(x=code(L), w=weight(L), y=mat(L, cols=6), grad=False, ws=BASE, n=1 << 40):
        return (lib.lm_linear8_grad if grad else lib.lm_linear8)(ref(x), ref(w), ref(y), ws, n, None)

    assert call(x=None) == INVALID and call(w=None) == INVALID and call(y=None) == INVALID
    assert call(x=code(L, fmt=0)) == DTYPE and call(x=code(L, fmt=5)) == DTYPE and call(y=mat(L, cols=6, dtype=2)) == DTYPE
    assert call(x=code(L, cols=9)) == INVALID and call(y=mat(L, cols=7)) == INVALID and call(y=mat(L, rows=5, cols=6)) == INVALID
    assert call(grad=True) == INVALID and call(x=code(L, cols=6), y=mat(L, cols=7), grad=True) == INVALID
    assert call(x=code(L, ld=24)) == ALIGN and call(w=weight(L, ld=8)) == ALIGN and call(w=weight(L, scales=BASE + 1)) == ALIGN
    n = 1 << 30
    assert call(x=code(L, rows=n, lds=n, ld=1024), y=mat(L, rows=n, cols=6)) == UNSUPPORTED
    assert call(x=code(L, rows=n, lds=n), w=weight(L, rows=1 << 20), y=mat(L, rows=n, cols=1 << 20)) == UNSUPPORTED
    assert call(x=code(L, rows=0), y=mat(L, rows=0, cols=6)) == 0
    assert call(w=weight(L, rows=0), y=mat(L, cols=0)) == 0
    need = lib.lm_linear8_workspace(ref(code(L, rows=1000, cols=4096)), ref(weight(L, rows=4096, cols=4096)), 0)
    if need:
        x, w = code(L, rows=1000, cols=4096, ld=4096, lds=1000), weight(L, rows=4096, cols=4096, ld=4096, lds=32)
        assert call(x=x, w=w, y=mat(L, rows=1000, cols=4096), n=need - 1) == INVALID
        assert call(x=x, w=w, y=mat(L, rows=1000, cols=4096), ws=None) == INVALID
        assert call(x=x, w=w, y=mat(L, rows=1000, cols=4096), ws=BASE + 16) == ALIGN
    assert lib.lm_linear8_workspace(None, None, 0) == 0


def test_rotary_refusals(L):
    lib = L.load_library()

    def heads(tokens=4, heads=2, dim=8, lt=None, lh=None, dtype=1, data=BASE):
        return L.LmHeads(data, tokens, heads, dim, heads * dim if lt is None else lt, dim if lh is None else lh, dtype)

    def call(grad=False, q=(), k=(), ws=BASE, n=1 << 20, **kw):
        a = L.LmQkRotaryArgs()
        a.q.x = a.q.y = a.q.dx = heads()
        for part, v in ((a.q, q), (a.k, k)):
            for name, x in dict(v).items():
                setattr(part, name, x)
        a.positions, a.table, a.table_rows, a.turned, a.norm, a.eps = BASE, BASE, 100, 8, 1, 1e-6
        for name, x in kw.items():
            setattr(a, name, x)
        return lib.lm_qk_rotary_grad(ctypes.byref(a), ws, n, None) if grad else lib.lm_qk_rotary(ctypes.byref(a), None)

    v = lambda n=8, dtype=1, data=BASE: L.LmTensor(data, 1, n, dtype)  # noqa: E731
    assert lib.lm_qk_rotary(None, None) == INVALID and lib.lm_qk_rotary_grad(None, None, 0, None) == INVALID
    for bad, want in ((heads(dtype=2), DTYPE), (heads(dtype=0), DTYPE), (heads(tokens=5), INVALID), (heads(heads=3), INVALID), (heads(dim=10), INVALID),
                      (heads(data=0), INVALID), (heads(data=BASE + 1), ALIGN), (heads(lh=4), INVALID), (heads(lt=8), INVALID), (heads(lt=0), INVALID),
                      (heads(lt=-16), INVALID), (heads(lt=1 << 61), UNSUPPORTED)):
        assert call(q={"x": bad}) == want
        assert call(True, q={"dx": bad}) == want
    assert call(True, q={"x": heads(tokens=5)}) == INVALID
    assert call(q={"y": heads(lt=32)}) == INVALID                               # over x, other strides
    assert call(True, q={"dx": heads(lt=32)}) == INVALID
    assert call(q={"x": heads(dim=2000), "y": heads(dim=2000, data=BASE * 2)}) == UNSUPPORTED
    three = dict(x=heads(heads=3), y=heads(heads=3), dx=heads(heads=3))
    assert call(k={**three, "x": heads(heads=3, tokens=3)}) == INVALID and call(k={**three, "y": heads(heads=3, dtype=0)}) == DTYPE
    for t in (-2, 3, 10):
        assert call(turned=t) == INVALID
    assert call(positions=None) == INVALID and call(table=None) == INVALID and call(table_rows=-1) == INVALID
    assert call(positions=BASE + 4) == ALIGN and call(table=BASE + 2) == ALIGN
    for e in (-1e-9, float("nan"), float("inf")):
        assert call(eps=e) == INVALID
    assert call(q={"weight": v(7)}) == INVALID and call(q={"weight": v(dtype=3)}) == DTYPE and call(q={"weight": v(data=BASE + 1)}) == ALIGN
    assert call(q={"weight": v()}, norm=0) == INVALID and call(True, q={"dweight": v()}, norm=0) == INVALID
    assert call(True, q={"dweight": v(9)}) == INVALID
    assert call(True, q={"dweight": v()}, n=8) == INVALID and call(True, q={"dweight": v()}, ws=None) == INVALID
    assert call(True, q={"dweight": v()}, ws=BASE + 8) == ALIGN
    none = dict(x=heads(tokens=0), y=heads(tokens=0), dx=heads(tokens=0))
    assert call(q=none) == 0 and call(True, q=none) == 0


def test_packed_structs_are_the_header_s(L):
    """The binding's packed bytes are the ctypes structs' (and so the header's)."""
    from paper_2605_19811_gb300 import training as T
    n = iter(range(1, 1000))
    take = lambda k: [next(n) for _ in range(k)]  # noqa: E731

    def tensor():
        return L.LmTensor(*take(3), 1)

    m = [L.LmMatrix(*take(4), 1) for _ in range(4)]
    flat = lambda x: [getattr(x, f) or 0 for f, _ in x._fields_]  # noqa: E731
    assert T._pack_matrix(*flat(m[0])) == bytes(m[0])
    c = L.LmCheckpoint8(*take(6), 1)
    assert T._pack_checkpoint8(*flat(c)) == bytes(c)
    w = L.LmWeight8(*take(6))
    assert T._pack_weight8(*flat(w)) == bytes(w)
    pointers = take(7)
    a = L.LmLinearLogprobArgs(m[0], m[1], *pointers, m[2], m[3], 1)
    assert T._pack_linear_logprob(*flat(m[0]), *flat(m[1]), *pointers, *flat(m[2]), *flat(m[3]), 1) == bytes(a)
    parts, fields = [], []
    for _ in range(2):
        heads = [L.LmHeads(*take(6), 1) for _ in range(3)]
        tensors = [tensor(), tensor()]
        parts.append(L.LmRotaryPart(*heads, *tensors))
        for x in heads + tensors:
            fields += flat(x)
    tail = (*take(3), 64, 1, 0, 1e-6)
    assert T._pack_qk_rotary(*fields, *tail) == bytes(L.LmQkRotaryArgs(*parts, *tail))


def test_binding_refusals(L):
    from paper_2605_19811_gb300 import training as T
    codes, scales = torch.zeros(130, 32, dtype=torch.uint8), torch.ones(2, 1)
    T.Weight8(codes, scales, 20)
    for c, s, n in ((codes, scales, 33), (codes, scales[:1], 20), (codes.t(), scales, 20), (codes, torch.ones(2, 0), 20)):
        with pytest.raises(ValueError):
            T.Weight8(c, s, n)
    with pytest.raises(TypeError):
        T.Weight8(codes.float(), scales, 20)
    with pytest.raises(TypeError):
        T.Weight8(codes, scales.double(), 20)
    x = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError):
        T._heads(x.transpose(1, 2), "q")
    with pytest.raises(ValueError):
        T._heads(torch.zeros(3, 4, 2, 8).transpose(0, 1), "q")
    with pytest.raises(TypeError):
        T._heads(x.half(), "q")
    with pytest.raises(ValueError):
        T._heads(torch.zeros(8), "q")
    assert T._heads(torch.zeros(3, 4, 50)[..., :16].unflatten(-1, (2, 8)), "q")[1:] == (12, 2, 8, 50, 8, 0)
    table = torch.zeros(10, 4, 2)
    for p, t, e in ((torch.zeros(4, dtype=torch.int32), table, TypeError), (torch.zeros(5, dtype=torch.int64), table, ValueError), (None, table, ValueError),
                    (torch.zeros(4, dtype=torch.int64), table.double(), TypeError), (torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8), ValueError)):
        with pytest.raises(e):
            T._rotary_tail(4, p, t, True, 1e-6, False)
    with pytest.raises(ValueError):
        T.qk_rotary_grad(x, None, None, None)                     # the norm's gradient reads q
    for kw in (dict(dims=7), dict(dims=8, base=0.0), dict(dims=8, factor=-1.0), dict(dims=8, original=100, low=4.0, high=1.0)):
        with pytest.raises(ValueError):
            T.rotary_frequencies(**kw)
    with pytest.raises(ValueError):
        T.linear_logprob(torch.zeros(2, 4), torch.zeros(3, 4), accumulate=True)


def test_results_over_each_other_are_refused(L):
    lib = L.load_library()

    def head(dh=mat(L, data=2 * BASE), dweight=mat(L, rows=10, data=3 * BASE)):
        a = L.LmLinearLogprobArgs()
        a.h, a.weight, a.targets, a.lse, a.g_logp, a.dh, a.dweight = mat(L, data=4 * BASE), mat(L, rows=10, data=5 * BASE), BASE, BASE, BASE, dh, dweight
        codes = set()
        for f in (lib.lm_linear_logprob, lib.lm_linear_logprob_grad):
            codes.add(f(ctypes.byref(a), BASE + 128, 1 << 40, None))
        return codes

    assert head() == {ALIGN}                                       # the workspace, after all else
    for at in (4, 5, 3):
        assert head(dh=mat(L, data=at * BASE)) == {INVALID}
    for at in (4, 5):
        assert head(dweight=mat(L, rows=10, data=at * BASE)) == {INVALID}

    def rotary(grad, at, dweight=(0, 0)):
        a = L.LmQkRotaryArgs()
        for part, first, w in ((a.q, 0, dweight[0]), (a.k, 3, dweight[1])):
            for i, name in enumerate(("x", "y", "dx")):
                setattr(part, name, L.LmHeads(at[first + i] * BASE, 4, 2, 8, 32 if i == 0 else 16, 8, 1))
            part.dweight = L.LmTensor(w * BASE, 1, 8, 1) if w else L.LmTensor()
        a.turned, a.norm, a.eps = 0, 1, 1e-6
        return lib.lm_qk_rotary_grad(ctypes.byref(a), BASE + 8, 1 << 40, None) if grad else lib.lm_qk_rotary(ctypes.byref(a), None)

    assert rotary(True, (1, 2, 3, 4, 5, 6), (7, 8)) == ALIGN       # the workspace
    assert rotary(True, (1, 2, 2, 4, 5, 5), (7, 8)) == ALIGN       # over dy
    assert rotary(True, (1, 2, 3, 4, 5, 6), (7, 7)) == INVALID
    assert rotary(True, (1, 2, 1, 4, 5, 6), (7, 8)) == INVALID     # over x, other strides
    for at in ((1, 2, 3, 4, 5, 3), (1, 2, 5, 4, 5, 6), (1, 2, 4, 4, 5, 6), (1, 2, 3, 4, 5, 2), (1, 2, 3, 4, 5, 1)):
        assert rotary(True, at, (7, 8)) == INVALID
    for at in ((1, 2, 3, 4, 2, 6), (1, 4, 3, 4, 5, 6), (1, 2, 3, 4, 1, 6)):
        assert rotary(False, at) == INVALID


def test_8_bit_results_over_inputs_are_refused(L):
    """Tiles are stored while others' operands are still read, blocks packed while others are."""
    lib = L.load_library()
    over = lambda st: st == INVALID and b"written over" in lib.lm_last_error()  # noqa: E731
    for grad in (False, True):
        f = lib.lm_linear8_grad if grad else lib.lm_linear8
        cols = 6 if grad else 8

        def call(y, rows=4):
            m = mat(L, rows=rows, cols=14 - cols, data=y * BASE)
            return f(ref(code(L, rows=rows, cols=cols, codes=2 * BASE, scales=3 * BASE)), ref(weight(L, codes=4 * BASE, scales=5 * BASE)), ref(m), BASE, 1 << 40, None)

        for at in (2, 3, 4, 5):
            assert over(call(at))
        assert not over(call(6)) and call(2, rows=0) == 0
    # an empty sum reads neither operand
    assert not over(lib.lm_linear8(ref(code(L, cols=0, codes=BASE, scales=BASE)), ref(weight(L, cols=0)), ref(mat(L, cols=6)), BASE, 1 << 40, None))
    for fn in (lambda w, c: lib.lm_weight8_pack(ref(w), ref(c), None), lambda w, c: lib.lm_weight8_unpack(ref(c), ref(w), None)):
        c = weight(L, codes=2 * BASE, scales=3 * BASE)
        assert over(fn(mat(L, rows=6, data=2 * BASE), c)) and over(fn(mat(L, rows=6, data=3 * BASE), c))
        assert not over(fn(mat(L, rows=6, data=4 * BASE), c))
