"""The language-model entry points without a device: refusals before any HIP
call, the binding's structure against the header, and its host arrays."""
import ctypes
import gc
import os
import subprocess

import pytest

from paper_2310_00967_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_sets_host_arrays_outlive_the_call(monkeypatch):
    seen = {}

    class Library:
        @staticmethod
        def micro_grads_init(out, count, tensors, sizes, types, stream):
            junk = [bytes(64) for _ in range(1000)]
            gc.collect()
            seen["at"] = [ctypes.cast(tensors, ctypes.POINTER(ctypes.c_uint64))[i] for i in range(count)]
            seen["sizes"] = [ctypes.cast(sizes, ctypes.POINTER(ctypes.c_int64))[i] for i in range(count)]
            seen["types"] = [ctypes.cast(types, ctypes.POINTER(ctypes.c_int32))[i] for i in range(count)]
            del junk
            return _lib.MICRO_OK

    monkeypatch.setattr(_lib, "load", lambda: Library)
    at, sizes, types = [4096 * (i + 1) for i in range(300)], [i + 7 for i in range(300)], [i % 3 for i in range(300)]
    _lib.micro_grads_init(at, sizes, types)
    assert (seen["at"], seen["sizes"], seen["types"]) == (at, sizes, types)


def test_structure_and_constants_match_the_header(tmp_path):
    names = ["MICRO_TYPE_F32", "MICRO_TYPE_F16", "MICRO_TYPE_BF16", "MICRO_IDS_I32", "MICRO_IDS_I64"]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "micro_sparsify.h"', "int main(void) {",
             'printf("size %zu\\n", sizeof(micro_table_config));']
    lines += [f'printf("{f} %zu\\n", offsetof(micro_table_config, {f}));' for f, _ in _lib.micro_table_config._fields_]
    lines += [f'printf("{n} %d\\n", (int)({n}));' for n in names] + ["return 0; }"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(_lib.micro_table_config)
    for f, _ in _lib.micro_table_config._fields_:
        assert int(got[f]) == getattr(_lib.micro_table_config, f).offset
    for n in names:
        assert int(got[n]) == getattr(_lib, n)


def test_default_configuration():
    c = _lib.default_table_config()
    assert (c.padding_id, c.ignored, c.score_bytes) == (-1, -100, 2 ** 31)


def test_calls_with_null_handles_are_refused():
    lib = _lib.load()
    one = ctypes.c_void_p(4096)
    assert lib.micro_grads_norm(None, one, None) == _lib.MICRO_EINVAL
    assert lib.micro_grads_clip(None, 1.0, None, None) == _lib.MICRO_EINVAL
    assert lib.micro_grads_flatten(None, 1.0, None, one, None) == _lib.MICRO_EINVAL
    assert lib.micro_table_lookup(None, one, 8, one, 0, 1, 1.0, one, 8) == _lib.MICRO_EINVAL
    assert lib.micro_table_lookup_grad(None, one, 8, one, 0, 1, 1.0, 0, one, 8) == _lib.MICRO_EINVAL
    assert lib.micro_table_loss(None, one, 8, one, 8, one, 0, 1, 0, one, one) == _lib.MICRO_EINVAL
    assert lib.micro_table_loss_grad(None, one, 8, one, 8, one, 0, 1, 0, 1.0, 0, one, one, one, 8, one, 8) == _lib.MICRO_EINVAL
    assert "NULL" in _lib.last_error()
    lib.micro_grads_free(None)
    lib.micro_table_free(None)
    lib.micro_table_config_default(None)


@pytest.mark.parametrize("addresses,sizes,types", [
    ([4096], [-1], [0]), ([4096], [5], [3]), ([4096], [5], [-1]), ([0], [5], [0]), ([4097], [5], [0]), ([4099], [5], [2]),
    ([4096, 4100], [2, 2], [0, 0]), ([4096, 1 << 20], [2 ** 60, 2 ** 62], [0, 0]), ([8192, 4096], [10, 4097], [0, 0])])
def test_tensor_lists_that_are_refused(addresses, sizes, types):
    with pytest.raises(_lib.MicroError) as e:
        _lib.micro_grads_init(addresses, sizes, types)
    assert e.value.status == _lib.MICRO_EINVAL


def test_set_and_table_arguments():
    lib = _lib.load()
    out = ctypes.c_void_p(1)
    assert lib.micro_grads_init(None, 0, None, None, None, None) == _lib.MICRO_EINVAL
    assert lib.micro_grads_init(ctypes.byref(out), 2, None, None, None, None) == _lib.MICRO_EINVAL
    assert out.value is None
    out = ctypes.c_void_p(1)
    assert lib.micro_grads_init(ctypes.byref(out), -1, None, None, None, None) == _lib.MICRO_EINVAL
    assert lib.micro_table_init(None, 10, 8, 4, 0, None, None) == _lib.MICRO_EINVAL
    for vocab, dim, tokens, kind, status in ((0, 8, 4, 0, _lib.MICRO_EINVAL), (10, 0, 4, 0, _lib.MICRO_EINVAL),
                                             (10, 8, -1, 0, _lib.MICRO_EINVAL), (10, 8, 4, 3, _lib.MICRO_EINVAL),
                                             (2 ** 31 - 1, 8, 4, 0, _lib.MICRO_ERANGE), (10, 65537, 4, 0, _lib.MICRO_ERANGE),
                                             (10, 8, 2 ** 22 + 1, 0, _lib.MICRO_ERANGE)):
        out = ctypes.c_void_p(1)
        assert lib.micro_table_init(ctypes.byref(out), vocab, dim, tokens, kind, None, None) == status
        assert out.value is None
    cfg = _lib.default_table_config()
    cfg.score_bytes = -1
    assert lib.micro_table_init(ctypes.byref(out), 10, 8, 4, 0, None, ctypes.byref(cfg)) == _lib.MICRO_EINVAL


def test_without_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    import paper_2310_00967_amd as micro
    with pytest.raises(RuntimeError):
        micro.GradientSet([])
    with pytest.raises(RuntimeError):
        micro.TokenTable(10, 8, 4)
    out = ctypes.c_void_p(1)
    assert _lib.load().micro_table_init(ctypes.byref(out), 10, 8, 4, 0, None, None) == _lib.MICRO_EHIP
    assert out.value is None
