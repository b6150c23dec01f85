"""The 4-bit matrices' and the token draw's entry points without a device:
refusals before any HIP call, sizes, and the binding's structures against the
header."""
import copy
import ctypes
import operator
import os
import pickle
import subprocess

import numpy as np
import pytest
import torch

from paper_2310_00967_amd import PackedMatrix, TokenTable, _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ERANGE = _lib.MICRO_EINVAL, _lib.MICRO_ERANGE


def test_structures_match_the_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "micro_sparsify.h"', "int main(void) {"]
    for st in (_lib.micro_sampling, _lib.micro_mx4_matrix):
        lines.append(f'printf("{st.__name__} %zu\\n", sizeof({st.__name__}));')
        lines += [f'printf("{st.__name__}.{f} %zu\\n", offsetof({st.__name__}, {f}));' for f, _ in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for st in (_lib.micro_sampling, _lib.micro_mx4_matrix):
        assert int(got[st.__name__]) == ctypes.sizeof(st)
        for f, _ in st._fields_:
            assert int(got[f"{st.__name__}.{f}"]) == getattr(st, f).offset


@pytest.mark.parametrize("rows,cols,want", [(0, 0, (0, 0)), (1, 1, (64, 4)), (3, 128, (192, 12)), (3, 129, (384, 24)),
                                            (2 ** 24, 2 ** 24, (2 ** 47, 2 ** 43)), (5, 0, (0, 0))])
def test_bytes(rows, cols, want):
    assert _lib.micro_mx4_bytes(rows, cols) == want


def test_sides_that_are_refused():
    for rows, cols, status in ((-1, 4, EINVAL), (4, -1, EINVAL), (2 ** 24 + 1, 4, ERANGE), (4, 2 ** 24 + 1, ERANGE)):
        with pytest.raises(_lib.MicroError) as e:
            _lib.micro_mx4_bytes(rows, cols)
        assert e.value.status == status
    one = ctypes.c_int64()
    assert _lib.load().micro_mx4_bytes(1, 1, None, ctypes.byref(one)) == EINVAL
    assert _lib.load().micro_mx4_bytes(1, 1, ctypes.byref(one), None) == EINVAL


def test_calls_with_null_handles_are_refused():
    lib = _lib.load()
    m = _lib.micro_mx4_matrix(4096, 8192, 1, 1)
    assert lib.micro_mx4_init(None, None) == EINVAL
    assert lib.micro_mx4_pack(None, 65536, 0, 1, 1, 1, m, None) == EINVAL
    assert lib.micro_mx4_unpack(None, m, 65536, 0, 1) == EINVAL
    assert lib.micro_mx4_product(None, m, m, 0, 65536, 0, 1) == EINVAL
    assert lib.micro_mx4_linear(None, 65536, 0, 1, m, m, 0, 131072, 0, 1) == EINVAL
    assert lib.micro_table_sample(None, 4096, 0, 1, 1, 4096, _lib.micro_sampling(), 8192, 1, None) == EINVAL
    assert "NULL" in _lib.last_error()
    lib.micro_mx4_free(None)


@pytest.fixture
def handle():
    """Memory in a handle's place: a refusal looks at none of it."""
    return ctypes.create_string_buffer(256)


def matrix(codes=1 << 20, scales=1 << 24, rows=10, cols=40):
    return _lib.micro_mx4_matrix(codes, scales, rows, cols)


@pytest.mark.parametrize("x,kind,stride,rows,cols,packed,turned,status", [
    (1 << 30, 0, 40, 10, 40, None, None, EINVAL), (1 << 30, 3, 40, 10, 40, matrix(), None, EINVAL),
    (1 << 30, 0, 39, 10, 40, matrix(), None, EINVAL), (0, 0, 40, 10, 40, matrix(), None, EINVAL),
    ((1 << 30) + 2, 0, 40, 10, 40, matrix(), None, EINVAL), (1 << 30, 0, 40, 10, 40, matrix(rows=11), None, EINVAL),
    (1 << 30, 0, 40, 10, 40, None, matrix(), EINVAL), (1 << 30, 0, 40, 10, 40, matrix(codes=0), None, EINVAL),
    (1 << 30, 0, 40, 10, 40, matrix(codes=(1 << 20) + 8), None, EINVAL),
    (1 << 30, 0, 40, 10, 40, matrix(scales=(1 << 24) + 2), None, EINVAL),
    (1 << 20, 0, 40, 10, 40, matrix(), None, EINVAL), (1 << 30, 0, 40, 10, 40, matrix(scales=1 << 20), None, EINVAL),
    (1 << 30, 0, 40, 10, 40, matrix(), matrix(rows=40, cols=10), EINVAL), (1 << 30, 0, 40, -1, 40, matrix(), None, EINVAL),
    (1 << 30, 0, (1 << 32) + 1, 10, 40, matrix(), None, EINVAL), (1 << 30, 0, 40, 2 ** 24 + 1, 40, matrix(), None, ERANGE)])
def test_packings_that_are_refused(handle, x, kind, stride, rows, cols, packed, turned, status):
    assert _lib.load().micro_mx4_pack(handle, x, kind, stride, rows, cols, packed, turned) == status


def test_products_that_are_refused(handle):
    lib = _lib.load()
    a, b = matrix(), matrix(codes=1 << 21, scales=1 << 25, rows=7)
    out, x = 1 << 30, 1 << 31
    for args in ((None, b, 0, out, 0, 7), (a, None, 0, out, 0, 7), (a, matrix(cols=41), 0, out, 0, 7), (a, b, 0, out, 0, 6),
                 (a, b, 0, out, 5, 7), (a, b, 0, out + 1, 2, 7), (a, b, 0, 0, 0, 7), (a, b, 0, 1 << 21, 0, 7),
                 (a, b, 0, 1 << 24, 0, 7), (a, matrix(codes=0), 0, out, 0, 7), (a, matrix(rows=2 ** 24 + 1), 0, out, 0, 2 ** 25)):
        assert lib.micro_mx4_product(handle, *args) in (EINVAL, ERANGE), args
        if args[0] is not None:
            assert lib.micro_mx4_linear(handle, x, 0, 40, *args) in (EINVAL, ERANGE), args
    assert lib.micro_mx4_linear(handle, x, 0, 39, a, b, 0, out, 0, 7) == EINVAL
    assert lib.micro_mx4_linear(handle, 1 << 20, 0, 40, a, b, 0, out, 0, 7) == EINVAL  # scratch over x
    assert lib.micro_mx4_linear(handle, x, 0, 40, a, a, 0, out, 0, 10) == EINVAL  # and over b
    assert lib.micro_mx4_linear(handle, out, 0, 40, a, b, 0, out, 0, 7) == EINVAL
    assert lib.micro_mx4_unpack(handle, a, out, 0, 39) == EINVAL
    assert lib.micro_mx4_unpack(handle, a, 1 << 20, 0, 40) == EINVAL


def test_packed_matrices_of_other_shapes_and_types_are_refused():
    u8 = torch.uint8
    m = PackedMatrix(torch.zeros(3, 3, 64, dtype=u8), torch.zeros(3, 3, 4, dtype=u8), 3, 300)
    assert m.shape == (3, 300) and m.device.type == "cpu"
    for codes, scales, error in ((torch.zeros(3, 192, dtype=u8), m.scales, ValueError), (m.codes, torch.zeros(2, 3, 4, dtype=u8), ValueError),
                                 (m.codes.char(), m.scales, TypeError), (torch.zeros(3, 64, 3, dtype=u8).transpose(1, 2), m.scales, TypeError),
                                 (m.codes, None, TypeError)):
        with pytest.raises(error):
            PackedMatrix(codes, scales, 3, 300)
    with pytest.raises(ValueError):
        PackedMatrix(m.codes, m.scales, -3, 300)


class Whole:
    """A whole number that is no int."""

    def __init__(self, value):
        self.value = value

    def __index__(self):
        return self.value


def test_a_whole_number_past_64_bits_is_refused_as_a_setting():
    """A ctypes structure takes one modulo 2^64."""
    table = TokenTable.__new__(TokenTable)  # a setting that is a number looks at no handle
    table._torch, table._tensor = torch, torch.Tensor
    s = _lib.micro_sampling()
    for top_k in (2 ** 63, 2 ** 64, 2 ** 64 + 5, -2 ** 63 - 1, 10 ** 400, Whole(2 ** 64 + 5), np.uint64(2 ** 64 - 1)):
        with pytest.raises(OverflowError, match="top_k"):
            table._setting(s, "top_k", top_k, torch.int32, 4)
        assert s.top_k == 0
    for top_k in (2 ** 63 - 1, -2 ** 63, 5):
        assert table._setting(s, "top_k", top_k, torch.int32, 4) is None and s.top_k == top_k
    for whole in (Whole(5), True, np.int64(5), np.uint8(5)):
        assert table._setting(s, "top_k", whole, torch.int32, 4) is None and s.top_k == int(operator.index(whole))
    for wrong in (2.5, "5", None, 5.0):
        with pytest.raises(TypeError):
            table._setting(s, "top_k", wrong, torch.int32, 4)
    with pytest.raises(OverflowError):
        table._setting(s, "temperature", 10 ** 400, torch.float32, 4)
    table._setting(s, "temperature", 2 ** 64, torch.float32, 4)
    assert s.temperature == 2.0 ** 64


def packed_on_the_cpu(rows=3, cols=300):
    groups = -(-cols // 128)
    gen = torch.Generator().manual_seed(rows)
    return PackedMatrix(torch.randint(256, (groups, rows, 64), generator=gen, dtype=torch.uint8),
                        torch.randint(255, (groups, rows, 4), generator=gen, dtype=torch.uint8), rows, cols)


def test_a_packed_matrix_is_one_state():
    """What the calls marshalled natively take and what the others do is the same,
    and stays so: its parts are not assigned."""
    m, other = packed_on_the_cpu(), packed_on_the_cpu(4, 300)
    for name in ("codes", "scales", "rows", "cols", "shape", "device"):
        with pytest.raises(AttributeError):
            setattr(m, name, getattr(other, name))
    assert m.shape == (m.rows, m.cols) == (3, 300)
    for same in (m, copy.copy(m), copy.deepcopy(m), pickle.loads(pickle.dumps(m))):
        codes, scales, rows, cols = same._parts
        assert codes is same.codes and scales is same.scales and (rows, cols) == (same.rows, same.cols)
        c = same._c
        assert (c.codes, c.scales, c.rows, c.cols) == (codes.data_ptr(), scales.data_ptr(), 3, 300)
        assert torch.equal(codes, m.codes) and torch.equal(scales, m.scales)
    assert copy.deepcopy(m).codes.data_ptr() != m.codes.data_ptr()


def changes_in_place():
    """What may happen to a matrix's tensors behind its back, and the error of a call
    that would read them."""
    return [(lambda m: m.codes.resize_(0), ValueError), (lambda m: m.scales.resize_(1, 1, 4), ValueError),
            (lambda m: m.codes.unsqueeze_(0), ValueError), (lambda m: m.codes.transpose_(0, 1), (TypeError, ValueError)),
            (lambda m: m.scales.set_(torch.zeros(2, dtype=torch.uint8, device=m.device)), ValueError),
            (lambda m: setattr(m.codes, "data", m.codes[:, :1].contiguous()), ValueError),
            (lambda m: setattr(m.codes, "data", m.codes.float()), TypeError)]


@pytest.mark.parametrize("change,error", changes_in_place())
def test_a_matrix_whose_tensors_were_changed_in_place_is_refused(change, error):
    m = packed_on_the_cpu()
    assert m._c.codes == m.codes.data_ptr()
    change(m)
    with pytest.raises(error):
        m._c  # noqa: B018

