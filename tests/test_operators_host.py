"""The operators' entry points without a GPU: bad arguments are refused with a code and a message before anything is
launched, what has nothing to do returns, and workspace sizes are those of the sizes alone."""
import ctypes
import math
import os

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


def test_layer_norm_refusals(lib):
    def call(x=P, x_stride=8, weight=P, bias=P, y=P, y_stride=8, mean=P, rstd=P, rows=2, cols=8, eps=1e-5, kind=FP32, weight_kind=FP32):
        return lib.mlda_layer_norm(x, x_stride, weight, bias, y, y_stride, mean, rstd, rows, cols, eps, kind, weight_kind, None)

    for bad in ({"rows": -1}, {"cols": 0}, {"cols": 2 ** 30 + 1}, {"kind": 3}, {"kind": -1}, {"kind": BF16, "weight_kind": FP16}, {"weight_kind": BF16},
                {"eps": -1e-9}, {"eps": math.nan}, {"eps": math.inf}, {"x": None}, {"y": None}, {"x_stride": 7}, {"y_stride": 7}, {"x": P + 2},
                {"x": P + 1, "kind": BF16}, {"y": P + 2}, {"weight": P + 2}, {"bias": P + 1}, {"mean": P + 2}, {"rstd": P + 2},
                {"y_stride": 9}):
        refused(lib, call(**bad), word="layer norm")
    assert call(rows=0, x=None, y=None) == 0


def test_layer_norm_backward_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.mlda_layer_norm_workspace_bytes(2, 8, ctypes.addressof(n)) == 0 and n.value > 0

    def call(g=P, g_stride=8, x=2 * P, x_stride=8, mean=P, rstd=P, weight=P, dx=3 * P, dx_stride=8, dw=P, db=P, rows=2, cols=8, kind=FP32,
             weight_kind=FP32, ws=P, size=n.value):
        return lib.mlda_layer_norm_backward(g, g_stride, x, x_stride, mean, rstd, weight, dx, dx_stride, dw, db, rows, cols, kind, weight_kind, ws, size, None)

    for bad in ({"rows": -1}, {"cols": 0}, {"kind": 7}, {"weight_kind": FP16}, {"g": None}, {"x": None}, {"mean": None}, {"rstd": None}, {"mean": P + 1},
                {"g_stride": 7}, {"x_stride": 3}, {"dx_stride": 5}, {"dx": P, "dx_stride": 9}, {"dx": 2 * P, "dx_stride": 9}, {"weight": P + 2},
                {"dw": P + 2}, {"db": P + 2}, {"ws": None}, {"ws": P + 2}):
        refused(lib, call(**bad), word="layer norm")
    refused(lib, call(size=n.value - 1), -2, "workspace")
    assert call(dx=None, dw=None, db=None, ws=None, size=0) == 0          # nothing is wanted
    assert call(rows=0, g=None, x=None, dw=None, db=None) == 0
    for bad in ((-1, 8), (2, 0)):
        refused(lib, lib.mlda_layer_norm_workspace_bytes(*bad, ctypes.addressof(n)))
    refused(lib, lib.mlda_layer_norm_workspace_bytes(2, 8, None), word="null")


def test_logprobs_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.mlda_token_logprobs_workspace_bytes(2, 50000, 5, FP32, ctypes.addressof(n)) == 0 and n.value > 0

    def forward(logits=P, stride=50000, rows=2, vocab=50000, kind=FP32, tokens=P, row_ptr=P, total=9, top=5, logprobs=P, stats=P, entropy=P,
                ids=P, top_logprobs=P, ws=P, size=n.value):
        return lib.mlda_token_logprobs(logits, stride, rows, vocab, kind, tokens, row_ptr, total, top, logprobs, stats, entropy, ids, top_logprobs, ws, size, None)

    def backward(logits=P, stride=50000, rows=2, vocab=50000, kind=FP32, tokens=P, row_ptr=P, total=9, stats=P, grad=P, entropy=P, grad_entropy=P,
                 out=2 * P, out_stride=50000):
        return lib.mlda_token_logprobs_backward(logits, stride, rows, vocab, kind, tokens, row_ptr, total, stats, grad, entropy, grad_entropy, out, out_stride, None)

    def both(logits=P, stride=50000, rows=2, vocab=50000, kind=FP32, tokens=P, row_ptr=P, total=9, weights=P, logprobs=P, out=2 * P, out_stride=50000,
             ws=P, size=n.value):
        return lib.mlda_token_logprobs_grad(logits, stride, rows, vocab, kind, tokens, row_ptr, total, weights, logprobs, out, out_stride, ws, size, None)

    shared = ({"logits": None}, {"logits": P + 2}, {"stride": 49999}, {"rows": -1}, {"vocab": 0}, {"vocab": 2 ** 30 + 1}, {"kind": 4}, {"tokens": None},
              {"total": -1}, {"total": 2 ** 31}, {"row_ptr": None})
    for bad in shared:
        for call in (forward, backward, both):
            refused(lib, call(**bad), word="log-probabilities")
    for bad in ({"top": -1}, {"top": 33}, {"top": 6, "vocab": 5}, {"logprobs": None}, {"ids": None}, {"top_logprobs": None}, {"ws": None}, {"ws": P + 4}):
        refused(lib, forward(**bad), word="log-probabilities")
    refused(lib, forward(size=n.value // 2), -2, "workspace")
    for bad in ({"stats": None}, {"grad": None}, {"entropy": None}, {"out": None}, {"out_stride": 49999}, {"out": P, "out_stride": 50001}, {"out": P + 2}):
        refused(lib, backward(**bad), word="log-probabilities")
    for bad in ({"weights": None}, {"logprobs": None}, {"out": None}, {"out_stride": 49999}, {"out": P, "out_stride": 50001}, {"ws": None}):
        refused(lib, both(**bad), word="log-probabilities")
    refused(lib, both(size=8), -2, "workspace")
    for call in (forward, backward, both):
        assert call(rows=0, logits=None) == 0
    for bad in ((-1, 5, 0, FP32), (1, 0, 0, FP32), (1, 5, 6, FP32), (1, 5, -1, FP32), (1, 50, 33, FP32), (1, 5, 0, 9)):
        refused(lib, lib.mlda_token_logprobs_workspace_bytes(*bad, ctypes.addressof(n)))
    refused(lib, lib.mlda_token_logprobs_workspace_bytes(1, 5, 0, FP32, None), word="null")


def test_clip_refusals(lib):
    n = ctypes.c_size_t()
    assert lib.mlda_grad_norm_workspace_bytes(2, ctypes.addressof(n)) == 0 and n.value > 0
    held = {}

    def lists(at, sizes, types):
        held["at"] = (ctypes.c_void_p * len(at))(*at)
        held["sizes"] = (ctypes.c_int64 * len(sizes))(*sizes)
        held["types"] = (ctypes.c_int32 * len(types))(*types)
        return held["at"], held["sizes"], held["types"]

    def clip(at=(P, P), to=(P, P), sizes=(4, 4), types=(FP32, BF16), count=2, most=1.0, norm=P, ws=P, size=n.value):
        a, s, t = lists(at, sizes, types)
        out = (ctypes.c_void_p * len(to))(*to) if to is not None else None
        return lib.mlda_clip_grads(a, out, s, t, count, most, norm, ws, size, None)

    for bad in ({"at": (P, None)}, {"at": (P + 2, P)}, {"at": (P, P + 1)}, {"to": (P, None)}, {"to": (P + 2, P)}, {"to": None}, {"sizes": (4, -1)},
                {"sizes": (2 ** 40 + 1, 4)}, {"types": (FP32, 3)}, {"count": -1}, {"most": -0.5}, {"most": math.nan}, {"norm": None}, {"norm": P + 2},
                {"ws": None}, {"ws": P + 4}):
        refused(lib, clip(**bad), word="gradients")
    refused(lib, clip(size=n.value - 1), -2, "workspace")
    a, s, t = lists((P,), (4,), (FP32,))
    for bad in ((None, s, t), (a, None, t), (a, s, None)):
        refused(lib, lib.mlda_grad_norm(*bad, 1, P, P, n.value, None), word="null")
    refused(lib, lib.mlda_grad_norm_workspace_bytes(-1, ctypes.addressof(n)))
    refused(lib, lib.mlda_grad_norm_workspace_bytes(1, None), word="null")


def test_workspaces_are_small(lib):
    n = ctypes.c_size_t()
    for rows, cols in ((1, 1), (10 ** 6, 1000), (10 ** 9, 16), (300000, 10000), (5, 2 ** 30)):
        assert lib.mlda_layer_norm_workspace_bytes(rows, cols, ctypes.addressof(n)) == 0
        assert 8 * cols <= n.value <= 1024 * 8 * cols
    for rows in (1, 100, 511, 512, 10 ** 7):
        assert lib.mlda_token_logprobs_workspace_bytes(rows, 141000, 32, BF16, ctypes.addressof(n)) == 0
        assert n.value <= 8 * rows + (64 * 512 * 288 if rows < 512 else 0)
    assert lib.mlda_grad_norm_workspace_bytes(10000, ctypes.addressof(n)) == 0 and n.value <= 2 << 20


def test_the_binding_wants_tensors_on_a_gpu():
    x = torch.zeros(2, 3)
    v = torch.zeros(2)
    tokens = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: operators.layer_norm(x), lambda: operators.layer_norm_backward(x, x, v, v), lambda: operators.token_logprobs(x, tokens),
                 lambda: operators.token_logprobs_backward(v, x, tokens, x), lambda: operators.token_logprobs_grad(x, tokens, v),
                 lambda: operators.grad_norm([x]), lambda: operators.clip_grads([x], 1.0), lambda: operators.layer_norm(None), lambda: operators.clip_grads([], 1.0)):
        with pytest.raises(ValueError):
            call()


def test_the_library_is_built_where_the_calls_on_tensors_cannot_be(tmp_path, monkeypatch, capsys):
    """The sampler's build needs hipcc alone, as before there were operators on tensors."""
    from paper_1803_04631_amd import _build
    stub = tmp_path / "hipcc"                        # writes its output and nothing else
    stub.write_text('#!/bin/sh\nwhile [ $# -gt 0 ]; do if [ "$1" = -o ]; then echo built > "$2"; fi; shift; done\n')
    stub.chmod(0o755)
    stale = tmp_path / "_tensors.so"
    stale.write_text("of another library")
    monkeypatch.setattr(_build, "LIB_PATH", str(tmp_path / "libmlda.so"))
    monkeypatch.setattr(_build, "TENSORS_PATH", str(stale))
    monkeypatch.setenv("HIPCC", str(stub))
    monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
    monkeypatch.setattr(_build, "_HERE", str(tmp_path))
    assert _build.build() == str(tmp_path / "libmlda.so")
    assert (tmp_path / "libmlda.so").read_text() == "built\n" and not stale.exists()
    assert "no-such-compiler" in capsys.readouterr().err
