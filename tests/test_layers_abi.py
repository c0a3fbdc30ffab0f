"""The layer operators' boundary without a GPU (include/layers/lsgd_layers.h):
every declared symbol is exported and bound, the header is plain C, sizes of
workspaces and pitches, and every refusal (each call here fails validation or
is a documented no-op, so nothing is ever launched)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "layers", "lsgd_layers.h")

# fake device addresses: only where no GPU is visible
pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake-pointer validation tests run only without a GPU")

L = pytest.importorskip("paper_1906_05936_amd._layers")
lib, pa = L.lib, L.ptr_array

OK, NULL, SIZE, GROUPS, ALIGN, DTYPE, HIP, ALIAS, UNSUPPORTED = range(9)
MB = 1 << 20
A, B, C, D, E = (MB * k for k in (1024, 2048, 3000, 4096, 5120))   # apart from each other
BIG = 1 << 31


def test_declared_exported_and_bound():
    names = set(re.findall(r"LSGD_API\s+[\w\s\*]+?\b(lsgd_\w+)\s*\(", open(HEADER).read()))
    assert names == set(L.EXPORTS)
    raw = ctypes.CDLL(L.lib._name)
    for name in names:
        assert hasattr(raw, name), name


def test_header_is_c99(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "layers/lsgd_layers.h"\n'
                   "int main(void) { return lsgd_pitch8(129) == 256 && lsgd_scale_pitch8(513) == 8 ? 0 : 1; }\n")
    lib_dir = os.path.dirname(L.lib._name)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    str(src), "-o", str(tmp_path / "h"), "-L" + lib_dir, "-llsgd", "-Wl,-rpath," + lib_dir], check=True)
    subprocess.run([str(tmp_path / "h")], check=True, timeout=60)


@pytest.mark.parametrize("cols", [0, 1, 127, 128, 129, 512, 513, 1024, 1025, 100003])
def test_pitches(cols):
    assert lib.lsgd_pitch8(cols) == L.pitch8(cols) == (cols + 127) // 128 * 128
    assert lib.lsgd_scale_pitch8(cols) == L.scale_pitch8(cols) == ((cols + 127) // 128 + 3) // 4 * 4


def lookup(table=A, tdt=0, rows=100, dim=64, tokens=B, it=1, n=10, scale=1.0, out=C, odt=0):
    return lib.lsgd_embed_lookup(table, tdt, rows, dim, tokens, it, n, scale, out, odt, None)


@pytest.mark.parametrize("bad,status", [
    (dict(tdt=2), DTYPE), (dict(odt=-1), DTYPE), (dict(it=2), DTYPE), (dict(rows=-1), SIZE), (dict(dim=BIG), SIZE),
    (dict(n=BIG), SIZE), (dict(n=-1), SIZE), (dict(rows=BIG - 1, dim=BIG - 1), SIZE), (dict(n=BIG - 1, dim=BIG - 1), SIZE),
    (dict(table=None), NULL), (dict(tokens=None), NULL), (dict(out=None), NULL), (dict(table=A + 8), ALIGN),
    (dict(out=C + 4), ALIGN), (dict(tokens=B + 4), ALIGN), (dict(tokens=B + 2, it=0), ALIGN), (dict(out=A), ALIAS),
    (dict(out=A + 100 * 64 * 4 - 16), ALIAS), (dict(tokens=C + 64), ALIAS),
    (dict(n=0, table=None, tokens=None, out=None), OK), (dict(dim=0, table=None, tokens=None, out=None), OK)])
def test_lookup(bad, status):
    assert lookup(**bad) == status


def grad(grads=(A,), gdt=0, tokens=(B,), it=1, workers=None, n=1500, rows=100, dim=64, out=C, odt=0, acc=0, ws=D, size=4 * MB):
    return lib.lsgd_embed_grad(None if grads is None else pa(grads), gdt, None if tokens is None else pa(tokens), it,
                               len(grads or ()) if workers is None else workers, n, rows, dim, 1.0, out, odt, acc, ws,
                               size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(gdt=3), DTYPE), (dict(odt=3), DTYPE), (dict(it=-1), DTYPE), (dict(workers=0), SIZE), (dict(workers=129), SIZE),
    (dict(n=-1), SIZE), (dict(n=BIG), SIZE), (dict(n=BIG // 2, workers=2), SIZE), (dict(rows=BIG), SIZE),
    (dict(rows=-1), SIZE), (dict(dim=-1), SIZE), (dict(dim=(1 << 24) + 1), SIZE), (dict(n=(1 << 28) + 1), SIZE), (dict(grads=None, workers=1), NULL),
    (dict(tokens=None), NULL), (dict(grads=(None,)), NULL), (dict(tokens=(None,)), NULL), (dict(out=None), NULL),
    (dict(ws=None), NULL), (dict(ws=D + 128), ALIGN), (dict(grads=(A + 8,)), ALIGN), (dict(tokens=(B + 4,)), ALIGN),
    (dict(out=C + 8), ALIGN), (dict(size=16), SIZE), (dict(out=A), ALIAS), (dict(ws=A), ALIAS), (dict(ws=B), ALIAS),
    (dict(ws=C), ALIAS), (dict(rows=0, out=None, grads=(None,), tokens=(None,), ws=None), OK),
    (dict(dim=0, out=None, grads=(None,), tokens=(None,), ws=None), OK), (dict(n=0, acc=1, grads=(None,)), OK)])
def test_grad(bad, status):
    assert grad(**bad) == status


def test_grad_workspace():
    size = ctypes.c_size_t()
    f = lib.lsgd_embed_grad_workspace_size
    for workers, n, rows, dim in [(1, 513, 1, 1), (1, 5, 1 << 20, 64), (1, 4096, 1000, 64), (2, 4096, 1 << 20, 100), (128, 70, 5, 5000)]:
        assert f(workers, n, rows, dim, ctypes.byref(size)) == OK
        assert size.value >= 8 * workers * n
        args = dict(grads=(A,) * workers, tokens=(B,) * workers, n=n, rows=rows, dim=dim, out=1 << 44, ws=1 << 45)
        assert grad(size=size.value - 1, **args) == SIZE
    for none in ((1, 0, 5, 5), (1, 5, 0, 5), (1, 5, 5, 0), (1, 512, 5, 5), (4, 128, 5, 5)):
        assert f(*none, ctypes.byref(size)) == OK and size.value == 0
    assert f(0, 1, 1, 1, ctypes.byref(size)) == SIZE and f(1, 1, 1, 1, None) == NULL


def quant(x=A, xdt=0, rows=10, cols=200, codes=B, scales=C):
    return lib.lsgd_quant8(x, xdt, rows, cols, codes, scales, None)


@pytest.mark.parametrize("bad,status", [
    (dict(xdt=2), DTYPE), (dict(rows=-1), SIZE), (dict(cols=BIG), SIZE), (dict(rows=BIG - 1, cols=BIG - 1), SIZE),
    (dict(x=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(x=A + 4), ALIGN),
    (dict(codes=B + 8), ALIGN), (dict(scales=C + 4), ALIGN), (dict(codes=A), ALIAS), (dict(scales=A + 16), ALIAS),
    (dict(scales=B + 10 * 256 - 16), ALIAS), (dict(rows=0, x=None), OK), (dict(cols=0, x=None), OK)])
def test_quant(bad, status):
    assert quant(**bad) == status


def copy_out(p=A, rows=200, cols=300, q=(B,), s=(C,), qt=(D,), st=(E,), n=None, nt=None):
    arr = lambda x: None if x is None else pa(x)  # noqa: E731
    return lib.lsgd_copy_out8(p, rows, cols, arr(q), arr(s), len(q or ()) if n is None else n, arr(qt), arr(st),
                              len(qt or ()) if nt is None else nt, None)


@pytest.mark.parametrize("bad,status", [
    (dict(n=-1), SIZE), (dict(n=129), SIZE), (dict(nt=129), SIZE), (dict(rows=-1), SIZE), (dict(cols=BIG), SIZE),
    (dict(rows=65535 * 128 + 1), SIZE), (dict(p=None), NULL), (dict(q=None, n=1), NULL), (dict(s=None), NULL),
    (dict(qt=None, nt=1), NULL), (dict(st=None), NULL), (dict(q=(None,)), NULL), (dict(st=(None,)), NULL),
    (dict(p=A + 4), ALIGN), (dict(q=(B + 8,)), ALIGN), (dict(s=(C + 1,)), ALIGN), (dict(qt=(D + 8,)), ALIGN),
    (dict(st=(E + 2,)), ALIGN), (dict(q=(A,)), ALIAS), (dict(qt=(B,)), ALIAS), (dict(q=(B, B), s=(C, C)), ALIAS),
    (dict(s=(A,)), ALIAS), (dict(rows=0, p=None), OK), (dict(cols=0, p=None), OK), (dict(q=(), s=(), qt=(), st=()), OK)])
def test_copy_out(bad, status):
    assert copy_out(**bad) == status


def matmul(a=A, sa=B, ab=1, m=10, b=C, sb=D, bb=128, n=20, k=300, out=E, odt=0):
    return lib.lsgd_matmul8(a, sa, ab, m, b, sb, bb, n, k, out, odt, None)


@pytest.mark.parametrize("bad,status", [
    (dict(odt=2), DTYPE), (dict(ab=2), UNSUPPORTED), (dict(bb=0), UNSUPPORTED), (dict(m=-1), SIZE), (dict(n=BIG), SIZE),
    (dict(k=-1), SIZE), (dict(m=BIG - 1, n=BIG - 1), SIZE), (dict(m=BIG - 1, k=BIG - 1), SIZE),
    (dict(n=BIG - 1, k=BIG - 1), SIZE), (dict(a=None), NULL), (dict(sa=None), NULL),
    (dict(b=None), NULL), (dict(sb=None), NULL), (dict(out=None), NULL), (dict(a=A + 8), ALIGN), (dict(sa=B + 4), ALIGN),
    (dict(b=C + 8), ALIGN), (dict(sb=D + 4), ALIGN), (dict(out=E + 8), ALIGN), (dict(out=A), ALIAS), (dict(out=B), ALIAS),
    (dict(out=C + 16), ALIAS), (dict(out=D), ALIAS), (dict(m=0, a=None, out=None), OK), (dict(n=0, b=None, out=None), OK)])
def test_matmul(bad, status):
    assert matmul(**bad) == status


def wgrad(g=A, x=B, s=C, m=1000, n=20, k=300, out=D, odt=0, acc=0, ws=E, size=64 * MB):
    return lib.lsgd_weight_grad8(g, x, s, m, n, k, out, odt, acc, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(odt=2), DTYPE), (dict(m=-1), SIZE), (dict(n=BIG), SIZE), (dict(k=-1), SIZE), (dict(m=BIG - 1, n=BIG - 1), SIZE),
    (dict(n=(1 << 24) + 1), SIZE), (dict(k=(1 << 24) + 1), SIZE), (dict(g=None), NULL), (dict(x=None), NULL), (dict(s=None), NULL),
    (dict(out=None), NULL), (dict(g=A + 8), ALIGN), (dict(x=B + 8), ALIGN), (dict(s=C + 4), ALIGN), (dict(out=D + 8), ALIGN),
    (dict(out=A), ALIAS), (dict(out=B), ALIAS), (dict(out=C), ALIAS), (dict(n=0, g=None, out=None), OK),
    (dict(k=0, x=None, out=None), OK), (dict(m=0, acc=1, g=None, out=None), OK)])
def test_weight_grad(bad, status):
    assert wgrad(**bad) == status


def test_weight_grad_workspace():
    size = ctypes.c_size_t()
    f = lib.lsgd_weight_grad8_workspace_size
    assert f(20000, 20, 300, ctypes.byref(size)) == OK and size.value > 0 and size.value % (20 * 300 * 4) == 0
    args = dict(m=20000, g=1 << 42, x=1 << 43, out=1 << 44, ws=1 << 45)
    assert wgrad(size=size.value - 1, **args) == SIZE
    assert wgrad(size=size.value, **dict(args, ws=None)) == NULL
    assert wgrad(size=size.value, **dict(args, ws=(1 << 45) + 64)) == ALIGN
    assert wgrad(size=size.value, **dict(args, ws=1 << 42)) == ALIAS
    assert f(0, 20, 300, ctypes.byref(size)) == OK and size.value == 0
    assert f(-1, 20, 300, ctypes.byref(size)) == SIZE and f(1, 1, 1, None) == NULL


def test_binding_refuses_before_the_call():
    """What the binding itself checks: devices, layouts, types, sizes."""
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU tensor"):
        L.embed_lookup(x, torch.zeros(2, dtype=torch.int64), x)
    with pytest.raises(ValueError, match="GPU tensor"):
        L.quant8(x, x, x)
    with pytest.raises(ValueError, match="GPU tensor"):
        L.matmul8(x, x, x, x, x)
    with pytest.raises(ValueError, match="at least one"):
        L.embed_grad([], [], _on_gpu(x))
    with pytest.raises(ValueError, match="block"):
        L.empty8(3, 4, 64, device="cpu")
    q, s = L.empty8(130, 600, 128, device="cpu")
    assert q.shape == (130, 640) and s.shape == (2, 8)


def _on_gpu(x):
    """A stand-in that passes the binding's look at the device only."""
    class Stand(torch.Tensor):
        @property
        def device(self):
            return torch.device("cuda", 0)
    return x.as_subclass(Stand)
