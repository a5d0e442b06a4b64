"""Callers that were compiled against an earlier header, without a GPU: what lies in their struct's padding is no field of it."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch  # noqa: F401  (first: where the library comes before it, it brings another HIP runtime than torch's into the process)

from paper_2602_16603_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _args(kv_dtype):
    # (valid but for kv_dtype; the weights are looked at by a task only)
    shape = B.fp_shape(1, 64, 1, 1, 64, 64, 1e-5, 1e4, B.FP_DTYPE_BF16, 16, 4, 16, 0, 0, kv_dtype)
    layers = (B.fp_layer_weights * 1)()
    for name, _ in B.fp_layer_weights._fields_:
        setattr(layers[0], name, 16)
    return C.byref(shape), layers, None


def test_the_struct_did_not_grow():
    """kv_dtype took the place of padding, so nothing behind an earlier caller's struct is read."""
    assert C.sizeof(B.fp_shape) == 64 and B.fp_shape.kv_dtype.offset == 60


@pytest.mark.parametrize("padding", [0, 1, 7, -1, 0x7f7f7f7f])
@pytest.mark.parametrize("call", ["symbol", "version 1"])
def test_padding_of_an_earlier_caller_is_not_read(padding, call):
    """... neither refused nor taken for an 8-bit cache: it gets as far as the device, or a model whose cache has no scales."""
    out = C.c_void_p()
    if call == "symbol":
        st = B.lib.fp_model_create(*_args(padding), C.byref(out))
    else:
        st = B.lib.fp_model_create_abi(*_args(padding), 1, C.byref(out))
    assert st != B.FP_ERR_INVALID, B.fp_last_error()
    if st == B.FP_OK:
        with pytest.raises(B.FlowPrefillError):
            B.fp_model_kv_scales(out.value)
        B.fp_model_destroy(out.value)


@pytest.mark.parametrize("version,kv_dtype,says", [(0, 0, "version"), (-1, 0, "version"), (B.FP_ABI_VERSION + 1, 0, "version"), (2, 7, "kv_dtype")])
def test_refused(version, kv_dtype, says):
    out = C.c_void_p()
    assert B.lib.fp_model_create_abi(*_args(kv_dtype), version, C.byref(out)) == B.FP_ERR_INVALID and says in B.fp_last_error()


@pytest.mark.parametrize("compiler,flags", [("gcc", ["-x", "c", "-std=c99"]), ("g++", ["-x", "c++", "-std=c++11"])])
def test_a_caller_of_this_header_says_its_version(compiler, flags, tmp_path):
    if shutil.which(compiler) is None or shutil.which("nm") is None:
        pytest.skip("no host compiler")
    obj = str(tmp_path / "caller.o")
    text = '#include "flowprefill.h"\nfp_status call(const fp_shape* s, const fp_layer_weights* l, fp_model** m) { return fp_model_create(s, l, 0, m); }\n'
    subprocess.run([compiler, *flags, "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", "-", "-o", obj],
                   input=text, text=True, check=True)
    undefined = subprocess.run(["nm", "-u", obj], stdout=subprocess.PIPE, text=True, check=True).stdout.split()
    assert "fp_model_create_abi" in undefined and "fp_model_create" not in undefined
