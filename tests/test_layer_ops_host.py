"""The layer operators' argument checks, before any device work (CPU): the C entry points through their argument
structures, and the binding's own checks.  No call here gets as far as a kernel."""
import ctypes

import pytest

import paper_2605_29489_gb300 as mp

A = 0x100000  # an aligned address, never touched
BAD = -1


def call(name, args, status=BAD):
    rc = getattr(mp.lib(), name)(ctypes.byref(args) if args is not None else None, None)
    assert rc == status, (name, rc, mp.mp_last_error())
    return mp.mp_last_error()


def norm(**k):
    d = dict(dtype=mp.MP_BF16, kind=mp.MP_NORM_LAYER, rows=4, cols=8, eps=1e-5, x=A, ldx=8, y=2 * A, ldy=8)
    return mp._NormArgs(**{**d, **k})


def norm_backward(**k):
    d = dict(dtype=mp.MP_BF16, kind=mp.MP_NORM_LAYER, rows=4, cols=8, dy=A, lddy=8, x=2 * A, ldx=8, dx=3 * A, lddx=8, mean=4 * A,
             rstd=5 * A)
    return mp._NormBackwardArgs(**{**d, **k})


def linear(**k):
    d = dict(dtype=mp.MP_BF16, act=mp.MP_ACT_NONE, rows=4, in_=16, out=8, x=A, ldx=16, w=2 * A, ldw=16, y=3 * A, ldy=8)
    return mp._LinearArgs(**{**d, **k})


def linear_backward(**k):
    d = dict(dtype=mp.MP_BF16, act=mp.MP_ACT_NONE, rows=4, in_=16, out=8, dy=A, lddy=8, x=2 * A, ldx=16, w=3 * A, ldw=16, dx=4 * A,
             lddx=16, dw=5 * A, lddw=16)
    return mp._LinearBackwardArgs(**{**d, **k})


@pytest.mark.parametrize("name", ["mp_norm", "mp_norm_backward", "mp_linear", "mp_linear_backward"])
def test_no_arguments(name):
    assert "NULL" in call(name, None)


def test_norm_refusals():
    assert "dtype" in call("mp_norm", norm(dtype=7))
    assert "kind" in call("mp_norm", norm(kind=2))
    assert "cols" in call("mp_norm", norm(cols=0))
    assert "cols" in call("mp_norm", norm(cols=(1 << 28) + 1))
    assert "rows" in call("mp_norm", norm(rows=1 << 49))
    for eps in (-1.0, float("nan"), float("inf")):
        assert "eps" in call("mp_norm", norm(eps=eps))
    assert "bias" in call("mp_norm", norm(kind=mp.MP_NORM_RMS, bias=A))
    assert "mean" in call("mp_norm", norm(kind=mp.MP_NORM_RMS, mean=A))
    assert "NULL" in call("mp_norm", norm(x=None))
    assert "row stride" in call("mp_norm", norm(ldx=7))
    assert "too large" in call("mp_norm", norm(rows=1 << 47, ldx=1 << 30, ldy=8))
    assert "aligned" in call("mp_norm", norm(x=A + 1))
    assert "device memory" in call("mp_norm", norm())
    call("mp_norm", norm(rows=0), mp.MP_OK)


def test_norm_backward_refusals():
    assert "weight is not" in call("mp_norm_backward", norm_backward(dweight=A))
    assert "dx is not" in call("mp_norm_backward", norm_backward(add=A, ldadd=8, dx=None, dbias=A))
    assert "mean" in call("mp_norm_backward", norm_backward(mean=None))
    assert "NULL" in call("mp_norm_backward", norm_backward(rstd=None))
    assert "bias" in call("mp_norm_backward", norm_backward(kind=mp.MP_NORM_RMS, mean=None, dbias=A))
    assert "device memory" in call("mp_norm_backward", norm_backward())
    call("mp_norm_backward", norm_backward(dx=None), mp.MP_OK)  # nothing is asked for


def test_linear_refusals():
    assert "dtype" in call("mp_linear", linear(dtype=-1))
    for act in (-1, 5):
        assert "activation" in call("mp_linear", linear(act=act))
    for k in (dict(in_=0), dict(out=0), dict(in_=1 << 31), dict(out=1 << 31)):
        assert "in and out" in call("mp_linear", linear(**k))
    assert "rows" in call("mp_linear", linear(rows=1 << 31))
    assert "NULL" in call("mp_linear", linear(w=None))
    assert "row stride" in call("mp_linear", linear(ldw=15))
    assert "device memory" in call("mp_linear", linear())
    call("mp_linear", linear(rows=0), mp.MP_OK)


def test_linear_backward_refusals():
    assert "mul is not" in call("mp_linear_backward", linear_backward(dmul=A, lddmul=8))
    assert "dx is not" in call("mp_linear_backward", linear_backward(dx_add=A, lddx_add=16, dx=None))
    assert "dw is not" in call("mp_linear_backward", linear_backward(dw_add=A, lddw_add=16, dw=None))
    assert "pre" in call("mp_linear_backward", linear_backward(act=mp.MP_ACT_SILU))
    assert "w is needed" in call("mp_linear_backward", linear_backward(w=None))
    assert "x is needed" in call("mp_linear_backward", linear_backward(x=None))
    assert "dy" in call("mp_linear_backward", linear_backward(dy=None))
    assert "device memory" in call("mp_linear_backward", linear_backward())
    call("mp_linear_backward", linear_backward(dx=None, dw=None), mp.MP_OK)


def test_structures_have_the_header_s_layout(tmp_path):
    """sizes and offsets of the binding's structures are those that a C compiler gives the header's"""
    import shutil
    import subprocess

    from paper_2605_29489_gb300 import build

    if shutil.which("gcc") is None:
        pytest.skip("gcc is not available")
    pairs = [(mp._NormArgs, "mp_norm_args"),
             (mp._NormBackwardArgs, "mp_norm_backward_args"), (mp._LinearArgs, "mp_linear_args"),
             (mp._LinearBackwardArgs, "mp_linear_backward_args")]
    lines, want = [], []
    for cls, name in pairs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        fields = [f[0] for f in cls._fields_]
        for f in fields:
            if f.startswith("ld") and f[2:] in fields:
                c = f[2:] + ".ld"
            elif "ld" + f in fields:
                c = f + ".data"
            else:
                c = {"in_": "in"}.get(f, f)
            lines.append(f'printf("%zu\\n", offsetof({name}, {c}));')
            want.append(getattr(cls, f).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"mergepipe.h\"\nint main(void) {\n" + "\n".join(lines) +
                   "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", build.INCLUDE, str(src), "-o", str(exe)])
    got = [int(v) for v in subprocess.check_output([str(exe)], text=True).split()]
    assert got == want


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 16), torch.zeros(8, 16)
    for f in (lambda: mp.mp_norm(x), lambda: mp.mp_linear(x, w), lambda: mp.mp_norm_backward(x, x, None, None, None),
              lambda: mp.mp_linear_backward(x[:, :8], x, w)):
        with pytest.raises(ValueError, match="GPU"):
            f()
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        mp.mp_norm(x.double())
