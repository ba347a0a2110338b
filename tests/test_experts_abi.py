"""The entry points of networks as experts without a GPU: exports, a C99 program, refusals; and the oracle's own pins."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import experts_oracle as XO

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "familyseer_experts.h")
LIB = os.path.join(ROOT, "paper_2201_00194_amd", "libfamilyseer.so")
EINVAL, EUNSUPPORTED = -1, -4


@pytest.fixture(scope="module")
def api():
    if not os.path.exists(LIB):
        from paper_2201_00194_amd import build
        build.build()
    from paper_2201_00194_amd import api as A
    return A


def test_library_exports_what_the_header_declares(api):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(fs_[a-z0-9_]+)\s*\(", src))
    assert {"fs_expert_matmul", "fs_expert_matmul_backward", "fs_quantize_rows", "fs_expert_gather_i8", "fs_expert_matmul_i8", "fs_distill",
            "fs_distill_backward"} <= names
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), n
        assert getattr(api._lib, n).argtypes is not None, n


def test_header_is_plain_c_and_links(api, tmp_path):
    src = tmp_path / "abi.c"
    src.write_text(r'''
#include <stdio.h>
#include <string.h>
#include "familyseer_experts.h"
int main(void) {
    fs_distill_params p;
    float x[8] = {0};
    memset(&p, 0, sizeof p);
    if (fs_distill(&p, 1, x, FS_F32, 8, NULL, FS_ID_I32, x, FS_F32, NULL, x, NULL, 0, NULL) != FS_EINVAL) return 1;
    if (strlen(fs_last_error()) == 0) return 2;
    if (fs_expert_matmul(-1, 1, 8, 8, x, FS_F32, 8, NULL, x, 8, 64, 0, x, FS_F32, 8, NULL) != FS_EINVAL) return 3;
    if (fs_expert_matmul_backward_workspace_bytes(1000000, 1, 64, 64, FS_BF16) == 0) return 4;
    if (fs_expert_matmul_backward_workspace_bytes(100, 1, 64, 64, FS_BF16) != 0) return 5;
    if (fs_quantize_rows(0, 4, NULL, FS_F16, 4, NULL, 4, NULL, NULL) != FS_OK) return 6;
    printf("ok %d %d %d\n", FS_MAX_I8_WIDTH, FS_MAX_CLASSES, FS_MAX_LISTED);
    return 0;
}
''')
    exe = tmp_path / "abi"
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe), "-L", os.path.dirname(LIB), "-lfamilyseer",
                    "-Wl,-rpath," + os.path.dirname(LIB)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    assert out == "ok %d %d %d\n" % (api.FS_MAX_I8_WIDTH, api.FS_MAX_CLASSES, api.FS_MAX_LISTED)


P = ctypes.c_void_p(4096)       # never dereferenced: every call below is refused
ODD = ctypes.c_void_p(4097)


def refused(api, code, word, rc):
    assert rc == code, (rc, api.fs_last_error())
    assert word in api.fs_last_error(), api.fs_last_error()


@pytest.mark.parametrize("at,value,code,word", [
    (0, -1, EINVAL, "slots"), (0, 1 << 31, EINVAL, "slots"), (1, 0, EINVAL, "n_experts"), (1, 1025, EUNSUPPORTED, "n_experts"), (2, 0, EINVAL, "width"),
    (2, 1048577, EUNSUPPORTED, "width"), (3, -4, EINVAL, "width"), (4, None, EINVAL, "x is NULL"), (4, ODD, EINVAL, "aligned"), (5, 3, EINVAL, "element type"),
    (6, 15, EINVAL, "stride"), (7, None, EINVAL, "first"), (7, ODD, EINVAL, "first"), (8, None, EINVAL, "w is NULL"), (8, ODD, EINVAL, "aligned"),
    (9, 15, EINVAL, "stride"), (10, -1, EINVAL, "matrix to matrix"), (10, 1 << 51, EINVAL, "matrix to matrix"), (11, 2, EINVAL, "turned"), (12, None, EINVAL, "y is NULL"),
    (13, 2, EINVAL, "another type"), (13, 7, EINVAL, "element type"), (14, 23, EINVAL, "stride"), (14, 1 << 41, EINVAL, "stride")])
def test_product_refuses_bad_arguments(api, at, value, code, word):
    args = [8, 2, 16, 24, P, 1, 16, P, P, 16, 384, 0, P, 0, 24, None]
    args[at] = value
    refused(api, code, word, api._lib.fs_expert_matmul(*args))


def test_turned_weights_have_other_rows(api):
    args = [8, 2, 16, 24, P, 1, 16, P, P, 16, 384, 1, P, 0, 24, None]
    refused(api, EINVAL, "stride", api._lib.fs_expert_matmul(*args))


@pytest.mark.parametrize("at,value,code,word", [
    (0, -1, EINVAL, "slots"), (1, 0, EINVAL, "n_experts"), (2, 0, EINVAL, "width"), (3, 0, EINVAL, "width"), (4, None, EINVAL, "d_y is NULL"), (5, 5, EINVAL, "element type"),
    (6, 23, EINVAL, "stride"), (7, None, EINVAL, "x is NULL"), (8, 15, EINVAL, "stride"), (9, None, EINVAL, "first"), (10, 2, EINVAL, "accumulate"),
    (11, None, EINVAL, "d_w is NULL"), (12, 2, EINVAL, "another type"), (13, 15, EINVAL, "stride"), (14, 383, EINVAL, "matrix to matrix"), (15, None, EINVAL, "work"),
    (15, ctypes.c_void_p(4100), EINVAL, "work"), (16, 100, EINVAL, "working memory")])
def test_gradient_of_the_weights_refuses_bad_arguments(api, at, value, code, word):
    args = [1000000, 2, 16, 24, P, 1, 24, P, 16, P, 0, P, 0, 16, 384, P, 1 << 40, None]
    args[at] = value
    refused(api, code, word, api._lib.fs_expert_matmul_backward(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, -1, "rows"), (0, 1 << 31, "rows"), (1, 0, "width"), (2, None, "x is NULL"), (2, ODD, "aligned"), (3, 9, "element type"), (4, 15, "stride"), (5, None, "q is NULL"),
    (6, 15, "stride"), (7, None, "scale"), (7, ctypes.c_void_p(4098), "scale")])
def test_quantizing_refuses_bad_arguments(api, at, value, word):
    args = [4, 16, P, 2, 16, P, 16, P, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_quantize_rows(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, -1, "tokens"), (1, 0, "k 0"), (1, 17, "k 17"), (2, 0, "n_experts"), (3, 0, "width"), (4, None, "x is NULL"), (5, 9, "element type"), (6, 15, "stride"),
    (7, None, "first"), (8, None, "place"), (9, None, "q is NULL"), (10, 15, "stride"), (11, None, "scale")])
def test_gathering_in_8_bits_refuses_bad_arguments(api, at, value, word):
    args = [4, 2, 8, 16, P, 0, 16, P, P, P, 16, P, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_expert_gather_i8(*args))


@pytest.mark.parametrize("at,value,code,word", [
    (0, -1, EINVAL, "slots"), (1, 0, EINVAL, "n_experts"), (2, 131073, EUNSUPPORTED, "131072"), (3, 0, EINVAL, "width"), (4, None, EINVAL, "q is NULL"), (5, 15, EINVAL, "stride"),
    (6, None, EINVAL, "scale"), (7, None, EINVAL, "first"), (8, None, EINVAL, "w is NULL"), (9, 15, EINVAL, "stride"), (10, -1, EINVAL, "matrix to matrix"),
    (11, None, EINVAL, "w_scale"), (11, ODD, EINVAL, "w_scale"), (12, None, EINVAL, "y is NULL"), (13, 3, EINVAL, "element type"), (14, 23, EINVAL, "stride")])
def test_product_in_8_bits_refuses_bad_arguments(api, at, value, code, word):
    args = [8, 2, 16, 24, P, 16, P, P, P, 16, 384, P, P, 1, 24, None]
    args[at] = value
    refused(api, code, word, api._lib.fs_expert_matmul_i8(*args))


DISTILL = dict(n_classes=64, k=8, temperature=1.0, scale=1.0)


@pytest.mark.parametrize("change,code,word", [
    (dict(n_classes=0), EINVAL, "n_classes"), (dict(n_classes=1048577), EUNSUPPORTED, "n_classes"), (dict(k=0), EINVAL, "k 0"), (dict(k=1025), EUNSUPPORTED, "k 1025"),
    (dict(temperature=0.0), EINVAL, "temperature"), (dict(temperature=-1.0), EINVAL, "temperature"), (dict(temperature=float("nan")), EINVAL, "temperature"),
    (dict(temperature=1e-40), EINVAL, "temperature"),
    (dict(temperature=float("inf")), EINVAL, "temperature"), (dict(scale=float("nan")), EINVAL, "scale"), (dict(scale=float("-inf")), EINVAL, "scale")])
def test_distillation_refuses_bad_parameters(api, change, code, word):
    p = api._FsDistillParams(**{**DISTILL, **change})
    refused(api, code, word, api._lib.fs_distill(p, 4, P, 0, 64, P, 0, P, 0, None, P, P, 1 << 40, None))
    refused(api, code, word, api._lib.fs_distill_backward(p, 4, P, 0, 64, P, 0, P, 0, None, P, None, P, 64, P, 1 << 40, None))
    assert api._lib.fs_distill_workspace_bytes(p, 4, 0) == 0


@pytest.mark.parametrize("at,value,word", [
    (0, None, "params"), (1, -1, "tokens"), (1, 1 << 31, "tokens"), (2, None, "logits is NULL"), (2, ODD, "aligned"), (3, 4, "element type"), (4, 63, "stride"), (5, None, "ids"),
    (5, ctypes.c_void_p(4098), "ids"), (6, 2, "type 2 of ids"), (7, None, "teacher"), (8, 9, "element type"), (9, ODD, "total"), (10, None, "loss"), (10, ODD, "loss")])
def test_distillation_refuses_bad_arguments(api, at, value, word):
    args = [api._FsDistillParams(**DISTILL), 4, P, 0, 64, P, 0, P, 0, None, P, P, 1 << 40, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_distill(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, None, "params"), (1, -1, "tokens"), (2, None, "logits is NULL"), (5, None, "ids"), (6, -1, "type -1 of ids"), (7, None, "teacher"), (10, None, "d_loss"), (11, ODD, "loss"),
    (12, None, "d_logits is NULL"), (13, 63, "stride")])
def test_distillations_gradient_refuses_bad_arguments(api, at, value, word):
    args = [api._FsDistillParams(**DISTILL), 4, P, 0, 64, P, 0, P, 0, None, P, None, P, 64, P, 1 << 40, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_distill_backward(*args))


def test_calls_on_nothing_need_no_gpu(api):
    lib = api._lib
    assert lib.fs_expert_matmul(0, 2, 16, 24, None, 1, 16, None, None, 16, 384, 0, None, 0, 24, None) == 0
    assert lib.fs_expert_matmul_i8(0, 2, 16, 24, None, 16, None, None, None, 16, 384, None, None, 1, 24, None) == 0
    assert lib.fs_quantize_rows(0, 16, None, 0, 16, None, 16, None, None) == 0
    assert lib.fs_expert_gather_i8(0, 2, 8, 16, None, 0, 16, None, None, None, 16, None, None) == 0
    p = api._FsDistillParams(**DISTILL)
    assert lib.fs_distill(p, 0, None, 0, 64, None, 0, None, 0, None, None, None, 0, None) == 0
    assert lib.fs_distill_backward(p, 0, None, 0, 64, None, 0, None, 0, None, None, None, None, 64, None, 0, None) == 0


def test_binding_refuses_tensors_that_do_not_fit(api):
    import torch
    plan = api.ExpertPlan(torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32))
    for call in (lambda: api.fs_expert_matmul(torch.zeros(8, 4), plan, torch.zeros(2, 3, 4)), lambda: api.fs_quantize_rows(torch.zeros(8, 4)),
                 lambda: api.fs_expert_gather_i8(torch.zeros(4, 4), plan), lambda: api.fs_distill(api.distill_params(4, 2), torch.zeros(3, 4), None, None)):
        with pytest.raises(api.FsError) as e:
            call()
        assert "GPU" in str(e.value)
    w = torch.zeros(2, 3, 8)
    assert api._weights(w, "w", 2, torch.float32)[1:] == (3, 8, 8, 24)
    assert api._weights(w[:, :, :5], "w", 2, torch.float32)[1:] == (3, 5, 8, 24)
    assert api._weights(w[:, :2], "w", 2, torch.float32)[1:] == (2, 8, 8, 24)
    assert api._weights(w[:1].expand(2, 3, 8), "w", 2, torch.float32)[1:] == (3, 8, 8, 0)
    assert api._weights(torch.zeros(1, 1, 8)[:, :, :3], "w", 1, torch.float32)[1:] == (1, 3, 3, 3)
    for bad in (w[0], w.half(), w.transpose(1, 2), w[:, :, ::2]):
        with pytest.raises(api.FsError):
            api._weights(bad, "w", 2, torch.float32)
    with pytest.raises(api.FsError):
        api._weights(w, "w", 3, torch.float32)
    q = torch.zeros(4, 8, dtype=torch.int8)
    assert api._bytes_matrix(q[:, :3], "q")[1] == 8 and api._bytes_matrix(q[:1, :3], "q")[1] == 3
    for bad in (q.float(), q[0], q.t()):
        with pytest.raises(api.FsError):
            api._bytes_matrix(bad, "q")
    with pytest.raises(api.FsError):
        api._bytes_matrix(q, "q", 7)
    with pytest.raises(api.FsError):
        api._bytes_matrix(q, "q", 8, 5)
    for name in ("n_classes", "k"):
        with pytest.raises(api.FsError) as e:
            api.distill_params(**{"n_classes": 8, "k": 2, name: (1 << 32) + 2})
        assert name in str(e.value)


# ---- the oracle's pins -------------------------------------------------------------------------------

def test_oracle_products_worked_out_by_hand():
    x, w = np.array([[1.0, 2.0], [3.0, -1.0], [5.0, 5.0]]), np.array([[[1.0, 1.0]], [[2.0, 0.5]]])
    y, size = XO.matmul(x, [0, 1, 2], w)
    assert y.tolist() == [[3.0], [5.5], [0.0]] and size.tolist() == [[3.0], [6.5], [0.0]]
    d, _ = XO.matmul_backward(np.array([[2.0], [1.0], [9.0]]), x, [0, 1, 2], 2)
    assert d.tolist() == [[[2.0, 4.0]], [[3.0, -1.0]]]
    assert XO.bounds([-3, 2, 99, 99], 5) == [(0, 2), (2, 5), (5, 5), (5, 5)]


def test_oracle_integers_worked_out_by_hand():
    q, s = XO.quantize(np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0], [1, np.nan, 2, 3], [np.inf, 0, 1, 2]]))
    assert q.tolist() == [[127, -64, 0, 2], [0] * 4, [0] * 4, [0] * 4]
    assert s[0] == 1 and s[1] == np.float32(2.0 ** -126) and np.isnan(s[2:]).all()


def test_oracle_distillation_worked_out_by_hand():
    x, log = np.log(np.array([[1.0, 1.0, 2.0, 4.0]])), np.log
    loss, _, grad, _ = XO.distill(x, np.array([[3, 2]]), np.log([[6.0, 2.0]]), d_loss=[1.0])
    assert abs(loss[0] - (0.75 * log(0.75 / 0.5) + 0.25 * log(0.25 / 0.25))) < 1e-15
    np.testing.assert_allclose(grad, [[0.125, 0.125, 0.0, -0.25]], atol=1e-15)
    loss, _, grad, _ = XO.distill(x, np.array([[3, 2]]), np.log([[6.0, 2.0]]), total=[log(10.0)], d_loss=[2.0])
    assert abs(loss[0] - (0.6 * log(0.6 / 0.5) + 0.2 * log(0.2 / 0.25) + 0.2 * log(0.2 / 0.25))) < 1e-15
    np.testing.assert_allclose(grad, [[0.05, 0.05, 0.1, -0.2]], atol=1e-15)


@pytest.mark.parametrize("rest", [False, True])
def test_oracle_distillation_gradient_against_differences(rest):
    rng = np.random.default_rng(0)
    x, ids, t = rng.standard_normal((3, 9)), np.array([[0, 3], [2, 1], [5, 5]]), rng.standard_normal((3, 2))
    total = np.array([3.0, 2.5, 2.6]) if rest else None
    _, _, grad, _ = XO.distill(x, ids, t, 0.7, 1.3, total, np.ones(3))
    for r in range(3):
        for c in range(9):
            h = np.zeros_like(x)
            h[r, c] = 1e-6
            d = (XO.distill(x + h, ids, t, 0.7, 1.3, total)[0] - XO.distill(x - h, ids, t, 0.7, 1.3, total)[0])[r] / 2e-6
            assert abs(d - grad[r, c]) < 1e-8
