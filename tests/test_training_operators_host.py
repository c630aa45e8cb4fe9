"""4-bit matrices, dropout and the policy loss without a GPU: bad arguments are refused with a code and a message before anything is launched, what
has nothing to do returns, workspace sizes are those of the sizes alone; and the division that the kernels use."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_1803_04631_amd as mlda
from paper_1803_04631_amd import operators

FP32, BF16, FP16 = 0, 1, 2
P = 4096                  # an address that nothing reads: every call below ends before a launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mlda.LIB_PATH):
        mlda.build()
    return mlda.load_library()


def refused(lib, rc, code=-1, word=None):
    assert rc == code, rc
    message = lib.mlda_last_error().decode()
    assert len(message) > 10 and (word is None or word in message), message


def test_quantize_refusals(lib):
    def quantize(x=P, stride=40, codes=P, scales=P, rows=2, cols=40, kind=FP32):
        return lib.mlda_mx_quantize(x, stride, codes, scales, rows, cols, kind, None)

    def dequantize(x=P, stride=40, codes=P, scales=P, rows=2, cols=40, kind=FP32):
        return lib.mlda_mx_dequantize(codes, scales, x, stride, rows, cols, kind, None)

    for call in (quantize, dequantize):
        for bad in ({"x": None}, {"x": P + 2}, {"x": P + 1, "kind": BF16}, {"stride": 39}, {"codes": None}, {"codes": P + 8}, {"scales": None}, {"rows": -1},
                    {"cols": 0}, {"cols": 2 ** 30 + 1}, {"kind": 3}, {"kind": -1}):
            refused(lib, call(**bad), word="4-bit")
        assert call(rows=0, x=None, codes=None, scales=None) == 0


@pytest.mark.parametrize("rows,cols", [(2 ** 62, 2 ** 20), (2 ** 63 - 1, 1), (2 ** 54 + 1, 1), (2 ** 31, 2 ** 24)])
def test_no_size_runs_over(lib, rows, cols):
    """More elements than any memory has, whose bytes 64 bits could not count."""
    n = ctypes.c_size_t(5)
    refused(lib, lib.mlda_mx_linear_workspace_bytes(rows, cols, ctypes.addressof(n)), word="4-bit")
    refused(lib, lib.mlda_mx_quantize(P, cols, P, P, rows, cols, FP32, None), word="4-bit")
    refused(lib, lib.mlda_mx_dequantize(P, P, P, cols, rows, cols, FP32, None), word="4-bit")
    refused(lib, lib.mlda_mx_linear(P, cols, P, P, None, 2 * P, 50, rows, cols, 50, FP32, FP32, FP32, P, 2 ** 63, None), word="4-bit")
    assert n.value == 5
    assert lib.mlda_mx_linear_workspace_bytes(2 ** 54 // cols, cols, ctypes.addressof(n)) == 0 and n.value >= 2 ** 53


def test_product_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.mlda_mx_linear_workspace_bytes(3, 40, ctypes.addressof(n)) == 0 and n.value == 0
    assert lib.mlda_mx_linear_workspace_bytes(33, 140, ctypes.addressof(n)) == 0 and n.value == 64 * 8 * 17

    def call(x=P, x_stride=140, codes=P, scales=P, bias=P, y=2 * P, y_stride=50, rows=33, cols=140, words=50, kind=FP32, out=FP32, bias_kind=FP32, ws=P, size=64 * 8 * 17):
        return lib.mlda_mx_linear(x, x_stride, codes, scales, bias, y, y_stride, rows, cols, words, kind, out, bias_kind, ws, size, None)

    for bad in ({"x": None}, {"x": P + 2}, {"x_stride": 139}, {"codes": None}, {"codes": P + 4}, {"scales": None}, {"bias": P + 2}, {"y": None}, {"y": P},
                {"y": P + 2}, {"y_stride": 49}, {"rows": -1}, {"cols": 0}, {"cols": 2 ** 24 + 1, "x_stride": 2 ** 25}, {"words": 0}, {"words": 2 ** 30 + 1}, {"kind": 3}, {"out": 3}, {"out": -1},
                {"out": BF16, "bias_kind": FP16}, {"bias_kind": BF16}, {"ws": None}, {"ws": P + 8}):
        refused(lib, call(**bad), word="4-bit")
    refused(lib, call(size=64 * 8 * 17 - 1), -2, "workspace")
    assert call(rows=0, x=None, y=None, ws=None, size=0) == 0
    for rows, cols in ((17, 1000), (64, 1000), (65, 1000), (2048, 133), (10 ** 6, 1537), (16, 2 ** 24)):
        assert lib.mlda_mx_linear_workspace_bytes(rows, cols, ctypes.addressof(n)) == 0
        assert rows * cols / 32 * 17 <= n.value <= (rows + 31) * (cols / 32 + 8) * 17
    for bad in ((-1, 5), (1, 0), (1, 2 ** 24 + 1)):
        refused(lib, lib.mlda_mx_linear_workspace_bytes(*bad, ctypes.addressof(n)))
    refused(lib, lib.mlda_mx_linear_workspace_bytes(1, 5, None), word="null")


@pytest.mark.parametrize("rows,cols,laid", [(1, 16384, False), (1, 16385, True), (16, 1024, False), (16, 1025, True), (15, 1088, False), (17, 32, True)])
def test_which_rows_need_room(lib, rows, cols, laid):
    """Up to 16 rows and 512 blocks are put into 4 bits where they are used."""
    n = ctypes.c_size_t()
    assert lib.mlda_mx_linear_workspace_bytes(rows, cols, ctypes.addressof(n)) == 0 and (n.value > 0) == laid


def test_dropout_refusals(lib):
    def call(x=P, x_stride=8, residual=None, residual_stride=0, y=2 * P, y_stride=8, rows=2, cols=8, p=0.1, dev_step=None, first_row=0, kind=FP32):
        return lib.mlda_dropout(x, x_stride, residual, residual_stride, y, y_stride, rows, cols, p, 1, 0, dev_step, first_row, kind, None)

    for bad in ({"x": None}, {"x": P + 2}, {"x_stride": 7}, {"residual": P + 1, "residual_stride": 8}, {"residual": 3 * P, "residual_stride": 7}, {"y": None},
                {"y": P + 2}, {"y_stride": 7}, {"y": P, "y_stride": 9}, {"residual": 2 * P, "residual_stride": 9}, {"rows": -1}, {"cols": 0}, {"cols": 2 ** 30 + 1},
                {"p": -1e-9}, {"p": 1.0000001}, {"p": math.nan}, {"dev_step": P + 4}, {"first_row": -1}, {"first_row": 2 ** 32 - 1}, {"first_row": 2 ** 62},
                {"rows": 2 ** 32 + 1}, {"kind": 9}):
        refused(lib, call(**bad), word="dropout")
    assert call(rows=0, x=None, y=None) == 0


def test_policy_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.mlda_policy_loss_workspace_bytes(2 ** 20, ctypes.addressof(n)) == 0 and 0 < n.value < 1 << 17

    def call(l=P, old=P, reference=P, advantages=P, weights=P, row_ptr=P, rows=5, total=2 ** 20, low=0.2, high=0.2, kl=0.1, sums=P, grad=P, ws=P, size=n.value):
        return lib.mlda_policy_loss(l, old, reference, advantages, weights, row_ptr, rows, total, low, high, kl, sums, grad, ws, size, None)

    for bad in ({"l": None}, {"l": P + 2}, {"old": None}, {"old": P + 1}, {"reference": None}, {"reference": P + 2}, {"advantages": None}, {"advantages": P + 2},
                {"weights": P + 2}, {"row_ptr": P + 4}, {"row_ptr": None}, {"rows": -1}, {"total": -1}, {"total": 2 ** 31}, {"low": -0.1}, {"low": 1.1},
                {"low": math.nan}, {"high": -0.1}, {"high": math.nan}, {"kl": math.inf}, {"kl": math.nan}, {"sums": None}, {"sums": P + 2}, {"grad": None},
                {"grad": P + 2}, {"ws": None}, {"ws": P + 4}):
        refused(lib, call(**bad), word="policy loss")
    refused(lib, call(size=n.value - 1), -2, "workspace")
    for bad in (-1, 2 ** 31):
        refused(lib, lib.mlda_policy_loss_workspace_bytes(bad, ctypes.addressof(n)))
    refused(lib, lib.mlda_policy_loss_workspace_bytes(5, None), word="null")


@pytest.mark.parametrize("total", [40, 2 ** 20])
def test_the_gradient_is_not_written_over_what_other_words_read(lib, total):
    n = ctypes.c_size_t()
    assert lib.mlda_policy_loss_workspace_bytes(total, ctypes.addressof(n)) == 0
    rows, far = 10, 2 ** 30
    l, advantages, row_ptr = 3 * far, far, 2 * far
    for grad in (advantages, advantages + 4 * rows - 4, advantages - 4 * total + 4, row_ptr, row_ptr + 8 * rows + 4, row_ptr - 4 * total + 4):
        refused(lib, lib.mlda_policy_loss(l, l, None, advantages, None, row_ptr, rows, total, 0.2, 0.2, 0.0, P, grad, P if n.value else None, n.value, None), word="advantages")


def test_the_binding_wants_tensors_on_a_gpu():
    x, v = torch.zeros(2, 40), torch.zeros(2)
    q = operators.Mx4(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.uint8), 40)
    for call in (lambda: operators.mx4_quantize(x), lambda: operators.mx4_quantize(None), lambda: operators.mx4_dequantize(q), lambda: operators.mx4_linear(x, q),
                 lambda: operators.mx4_linear(x, None), lambda: operators.dropout(x, 0.1, 1), lambda: operators.dropout_backward(x, 0.1, 1),
                 lambda: operators.policy_loss(v, v, v)):
        with pytest.raises(ValueError):
            call()


def test_division(tmp_path):
    """Quotients for every kind of divisor, at the numbers beside multiples of it."""
    source = tmp_path / "divide.cpp"
    source.write_text(r'''
#include <cstdint>
#include <cstdio>
#define __device__
#define __forceinline__ inline
static uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
#include "divisor.hpp"
int main() {
    uint64_t wrong = 0, done = 0;
    auto check = [&](uint32_t by) {
        const mlda::Divisor d = mlda::divisor(by);
        const uint64_t most = (1ull << 31) - 1;
        for (int k = 0; k < 400; ++k) {
            const uint64_t multiple = (k < 200 ? (uint64_t)k : most / by - (k - 200)) * by;
            for (int64_t n = (int64_t)multiple - 1; n <= (int64_t)multiple + 1; ++n)
                if (n >= 0 && n <= (int64_t)most) { ++done; wrong += d((uint32_t)n) != (uint32_t)n / by; }
        }
    };
    for (uint32_t by = 1; by < 5000; ++by) check(by);
    for (int l = 12; l < 31; ++l) for (int64_t by = (1ll << l) - 3; by <= (1ll << l) + 3; ++by) if (by < (1ll << 31)) check((uint32_t)by);
    for (uint32_t by = 5001; by < (1u << 30); by += by / 3 + 1) check(by);
    printf("%llu %llu\n", (unsigned long long)wrong, (unsigned long long)done);
}
''')
    csrc = os.path.join(os.path.dirname(mlda.__file__), "csrc")
    empty = tmp_path / "hip"
    empty.mkdir()
    (empty / "hip_runtime.h").write_text("")
    program = tmp_path / "divide"
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", str(tmp_path), "-I", csrc, "-o", str(program), str(source)], check=True)
    wrong, done = map(int, subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split())
    assert wrong == 0 and done > 1_000_000
