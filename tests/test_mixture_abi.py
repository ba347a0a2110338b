"""The mixture entry points without a GPU: exports, a C99 program, refusals; and the oracle's own pins."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import mixture_oracle as MO

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "familyseer_mixture.h")
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
    assert {"fs_route", "fs_route_backward", "fs_expert_plan", "fs_expert_gather", "fs_expert_combine",
            "fs_expert_combine_backward", "fs_embed", "fs_embed_backward"} <= names
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), n
        assert hasattr(api._lib, n)


def test_header_is_plain_c_and_links(api, tmp_path):
    src = tmp_path / "abi.c"
    src.write_text(r'''
#include <stdio.h>
#include <string.h>
#include "familyseer_mixture.h"
int main(void) {
    fs_route_params p;
    float x[8] = {0};
    memset(&p, 0, sizeof p);
    if (fs_route(&p, 1, x, FS_F32, 8, NULL, NULL, NULL, NULL) != FS_EINVAL) return 1;
    if (strlen(fs_last_error()) == 0) return 2;
    if (fs_expert_plan_workspace_bytes(-1, 1, 1) != 0) return 3;
    if (fs_expert_plan_workspace_bytes(100000, 2, 8) == 0) return 4;
    if (fs_embed_backward_workspace_bytes(100, 8, FS_F32, 10, 2) == 0) return 5;
    printf("ok %d\n", FS_MAX_EXPERTS);
    return 0;
}
''')
    exe = tmp_path / "abi"
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe), "-L", os.path.dirname(LIB), "-lfamilyseer",
                    "-Wl,-rpath," + os.path.dirname(LIB)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout == "ok 1024\n"


P = ctypes.c_void_p(4096)       # never dereferenced: every call below is refused


def refused(api, code, word, rc):
    assert rc == code, (rc, api.fs_last_error())
    assert word in api.fs_last_error(), api.fs_last_error()


ROUTE = dict(n_experts=8, k=2, score=0, renormalise=1, n_groups=1, top_groups=1, group_best=1, scale=1.0)


@pytest.mark.parametrize("change,code,word", [
    (dict(n_experts=0), EINVAL, "n_experts"), (dict(n_experts=1025), EUNSUPPORTED, "n_experts"), (dict(k=0), EINVAL, "k 0"),
    (dict(k=9), EINVAL, "k 9"), (dict(n_experts=64, k=17), EUNSUPPORTED, "k 17"), (dict(score=2), EINVAL, "score"),
    (dict(renormalise=2), EINVAL, "renormalise"), (dict(n_groups=3), EINVAL, "groups"), (dict(n_groups=0), EINVAL, "groups"),
    (dict(n_groups=16), EINVAL, "groups"), (dict(n_groups=2, top_groups=3), EINVAL, "top_groups"), (dict(top_groups=0), EINVAL, "top_groups"),
    (dict(group_best=3), EINVAL, "group_best"), (dict(scale=float("nan")), EINVAL, "scale"), (dict(scale=float("inf")), EINVAL, "scale")])
def test_route_refuses_bad_parameters(api, change, code, word):
    p = api._FsRouteParams(**{**ROUTE, **change})
    lib = api._lib
    refused(api, code, word, lib.fs_route(p, 4, P, 0, 64, None, P, P, None))
    refused(api, code, word, lib.fs_route_backward(p, 4, P, 0, 64, P, P, P, 64, None))


@pytest.mark.parametrize("at,value,word", [
    (1, -1, "tokens"), (1, 1 << 30, "tokens"), (1, 1 << 62, "tokens"), (2, None, "logits is NULL"), (2, ctypes.c_void_p(4097), "aligned"),
    (3, 3, "element type"), (4, 7, "stride"), (4, -8, "stride"), (5, ctypes.c_void_p(4098), "bias"), (6, None, "expert"),
    (7, None, "weight"), (7, ctypes.c_void_p(4097), "weight")])
def test_route_refuses_bad_arguments(api, at, value, word):
    args = [api._FsRouteParams(**ROUTE), 4, P, 0, 8, None, P, P, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_route(*args))


def test_route_refuses_missing_parameters(api):
    refused(api, EINVAL, "params", api._lib.fs_route(None, 4, P, 0, 8, None, P, P, None))
    refused(api, EINVAL, "params", api._lib.fs_route_backward(None, 4, P, 0, 8, P, P, P, 8, None))


@pytest.mark.parametrize("at,value,word", [
    (1, -1, "tokens"), (2, None, "logits is NULL"), (3, -1, "element type"), (5, None, "expert"), (6, None, "d_weight"),
    (7, None, "d_logits"), (7, ctypes.c_void_p(4097), "d_logits"), (8, 7, "stride")])
def test_route_backward_refuses_bad_arguments(api, at, value, word):
    args = [api._FsRouteParams(**ROUTE), 4, P, 0, 8, P, P, P, 8, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_route_backward(*args))


@pytest.mark.parametrize("at,value,code,word", [
    (0, -1, EINVAL, "tokens"), (0, 1 << 31, EINVAL, "tokens"), (1, 0, EINVAL, "k 0"), (1, 17, EINVAL, "k 17"), (2, 0, EINVAL, "n_experts"),
    (2, 1025, EUNSUPPORTED, "n_experts"), (3, None, EINVAL, "expert"), (4, None, EINVAL, "first"), (5, None, EINVAL, "order"),
    (6, None, EINVAL, "place"), (7, None, EINVAL, "work"), (7, ctypes.c_void_p(4100), EINVAL, "work"), (8, 0, EINVAL, "working memory")])
def test_plan_refuses_bad_arguments(api, at, value, code, word):
    args = [100000, 2, 8, P, P, P, P, P, 1 << 30, None]
    args[at] = value
    refused(api, code, word, api._lib.fs_expert_plan(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, -1, "tokens"), (1, 0, "k 0"), (2, 0, "n_experts"), (3, 0, "width"), (4, None, "x is NULL"), (5, 9, "element type"),
    (6, 15, "stride"), (7, None, "first"), (8, None, "place"), (9, None, "xs is NULL"), (10, 15, "stride")])
def test_gather_refuses_bad_arguments(api, at, value, word):
    args = [4, 2, 8, 16, P, 0, 16, P, P, P, 16, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_expert_gather(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, 1 << 31, "tokens"), (1, 17, "k 17"), (2, 0, "width"), (3, None, "y is NULL"), (4, 9, "element type"), (5, 15, "stride"),
    (6, None, "place"), (7, ctypes.c_void_p(4097), "weight"), (8, None, "out is NULL"), (9, 15, "stride")])
def test_combine_refuses_bad_arguments(api, at, value, word):
    args = [4, 2, 16, P, 0, 16, P, P, P, 16, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_expert_combine(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, -1, "tokens"), (1, 0, "k 0"), (2, 0, "n_experts"), (3, 0, "width"), (4, None, "d_out is NULL"), (5, 9, "element type"),
    (6, 15, "stride"), (7, None, "y is NULL"), (8, 15, "stride"), (9, None, "first"), (10, None, "place"), (11, None, "weight"),
    (12, None, "d_y is NULL"), (13, 15, "stride"), (14, None, "d_weight")])
def test_combine_backward_refuses_bad_arguments(api, at, value, word):
    args = [4, 2, 8, 16, P, 0, 16, P, 16, P, P, P, P, 16, P, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_expert_combine_backward(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, 0, "n_vocab"), (0, 2147483647, "n_vocab"), (1, 0, "width"), (2, None, "table is NULL"), (3, 9, "element type"), (4, 15, "stride"),
    (5, -1, "rows"), (5, 1 << 31, "rows"), (6, 0, "n_cols"), (6, 1 << 29, "rows"), (7, None, "ids"), (7, ctypes.c_void_p(4097), "ids"),
    (8, 3, "type 3 of ids"), (9, ctypes.c_void_p(4097), "col_base"), (10, float("nan"), "scale"), (11, None, "out is NULL"),
    (12, 9, "element type"), (12, 2, "another type"), (13, 15, "stride")])
def test_embed_refuses_bad_arguments(api, at, value, word):
    args = [100, 16, P, 1, 16, 4, 3, P, 0, P, 1.0, P, 0, 16, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_embed(*args))


@pytest.mark.parametrize("at,value,word", [
    (0, 0, "n_vocab"), (1, 0, "width"), (2, None, "d_out is NULL"), (3, 9, "element type"), (4, 15, "stride"), (5, -1, "rows"),
    (6, 0, "n_cols"), (7, None, "ids"), (8, 3, "type 3 of ids"), (9, ctypes.c_void_p(4097), "col_base"), (10, float("inf"), "scale"),
    (11, 2, "accumulate"), (12, None, "d_table is NULL"), (13, 2, "another type"), (14, 15, "stride"), (15, None, "work"),
    (15, ctypes.c_void_p(4104), "work"), (16, 100, "working memory")])
def test_embed_backward_refuses_bad_arguments(api, at, value, word):
    args = [100, 16, P, 1, 16, 4, 3, P, 0, P, 1.0, 0, P, 0, 16, P, 1 << 30, None]
    args[at] = value
    refused(api, EINVAL, word, api._lib.fs_embed_backward(*args))


def test_calls_on_nothing_need_no_gpu(api):
    lib = api._lib
    p = api._FsRouteParams(**ROUTE)
    assert lib.fs_route(p, 0, None, 0, 8, None, None, None, None) == 0
    assert lib.fs_route_backward(p, 0, None, 0, 8, None, None, None, 8, None) == 0
    assert lib.fs_expert_gather(0, 2, 8, 16, None, 0, 16, None, None, None, 16, None) == 0
    assert lib.fs_expert_combine(0, 2, 16, None, 0, 16, None, None, None, 16, None) == 0
    assert lib.fs_embed(100, 16, P, 0, 16, 0, 1, None, 0, None, 1.0, None, 0, 16, None) == 0
    assert lib.fs_expert_plan_workspace_bytes(0, 2, 8) == 0


def test_binding_refuses_tensors_that_do_not_fit(api):
    import torch
    plan = api.ExpertPlan(torch.zeros(9, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32))
    for call in (lambda: api.fs_route(api.route_params(8, 2), torch.zeros(4, 8)),
                 lambda: api.fs_expert_gather(torch.zeros(4, 3), plan), lambda: api.fs_embed(torch.zeros(4, 4), torch.zeros(2).int())):
        with pytest.raises(api.FsError) as e:
            call()
        assert "GPU" in str(e.value)
    for bad in (torch.zeros(4, 8, dtype=torch.float64), torch.zeros(8), torch.zeros(8, 4).t()):
        with pytest.raises(api.FsError):
            api._matrix(bad, "x")
    with pytest.raises(api.FsError):
        api._matrix(torch.zeros(4, 8), "x", width=7)
    with pytest.raises(api.FsError):
        api._array(torch.zeros(4), "w", 4, torch.int32)
    with pytest.raises(api.FsError):
        api._array(torch.zeros(8)[::2], "w", 4, torch.float32)
    with pytest.raises(api.FsError):
        api._id_array(torch.zeros(2, 2, 2).int(), None)
    with pytest.raises(api.FsError):
        api._id_array(torch.zeros(4, 4).int().t(), None)


# ---- the oracle's pins -------------------------------------------------------------------------------


def test_oracle_route_on_a_token_worked_out_by_hand():
    x = np.array([[np.log(1.0), np.log(4.0), np.log(3.0), np.log(2.0)]])
    e, w = MO.route(x, 2, renormalise=False)
    assert e.tolist() == [[1, 2]]
    np.testing.assert_allclose(w, [[0.4, 0.3]], rtol=1e-14)
    e, w = MO.route(x, 2, renormalise=True, scale=7.0)
    np.testing.assert_allclose(w, [[4.0, 3.0]], rtol=1e-14)
    e, w = MO.route(x, 2, bias=[0.35, 0, 0, 0.25], renormalise=False)      # keys .45 .4 .3 .45
    assert e.tolist() == [[0, 3]]
    np.testing.assert_allclose(w, [[0.1, 0.2]], rtol=1e-14)
    y = np.array([[0.0, 3.0, 2.0, 2.5]])                                   # the second group has more, the first the best
    assert MO.route(y, 2, score="sigmoid", n_groups=2, group_best=2)[0].tolist() == [[3, 2]]
    assert MO.route(y, 2, score="sigmoid", n_groups=2, group_best=1)[0].tolist() == [[1, 0]]
    assert MO.route(np.ones((1, 4)), 2, n_groups=2)[0].tolist() == [[0, 1]]
    e, w = MO.route(np.array([[-np.inf, np.nan, 0.0, -np.inf]]), 2, score="sigmoid", renormalise=False)
    assert e.tolist() == [[2, -1]] and w.tolist() == [[0.5, 0.0]]
    e, w = MO.route(np.full((1, 4), -np.inf), 2)
    assert e.tolist() == [[-1, -1]] and w.tolist() == [[0, 0]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_oracle_route_gradient_against_differences(score, renormalise):
    rng = np.random.default_rng(5)
    x, dw = rng.standard_normal((3, 9)), rng.standard_normal((3, 4))
    kw = dict(score=score, renormalise=renormalise, scale=1.7)
    e, _ = MO.route(x, 4, **kw)

    def loss(z):
        total = 0.0
        for t in range(3):
            a = MO.log_scores(z[t], score)[e[t]]
            w = np.exp(a) / (np.sum(np.exp(a)) if renormalise else 1.0) * 1.7
            total += np.dot(w, dw[t])
        return total

    d, _ = MO.route_backward(x, e, dw, **kw)
    for t in range(3):
        for i in range(9):
            h = np.zeros_like(x)
            h[t, i] = 1e-6
            assert abs((loss(x + h) - loss(x - h)) / 2e-6 - d[t, i]) < 1e-8


def test_oracle_plan_gather_and_combine_fit_each_other():
    rng = np.random.default_rng(6)
    expert = rng.integers(-1, 5, (40, 3)).astype(np.int32)
    first, order, place = MO.plan(expert, 5)
    flat = expert.reshape(-1)
    assert first[-1] == np.sum(flat >= 0) and np.all(order[first[-1]:] == -1)
    for e in range(5):
        mine = order[first[e]: first[e + 1]]
        assert np.all(flat[mine] == e) and np.all(np.diff(mine) > 0)
        assert np.array_equal(place.reshape(-1)[mine], np.arange(first[e], first[e + 1]))
    x, g = rng.standard_normal((40, 4)), rng.standard_normal((120, 4))
    xs = MO.gather(x, order, 3)
    back, _ = MO.combine(g, place)
    assert abs(np.sum(xs * g) - np.sum(x * back)) < 1e-10                  # one is the other's transpose
    w, dout = rng.standard_normal((40, 3)), rng.standard_normal((40, 4))
    d_y, d_w, _ = MO.combine_backward(dout, g, place, w)
    out, _ = MO.combine(g, place, w)
    assert abs(np.sum(d_y * g) - np.sum(dout * out)) < 1e-10
    assert abs(np.sum(d_w * w) - np.sum(dout * out)) < 1e-10


def test_oracle_embedding_is_a_product_with_counts():
    rng = np.random.default_rng(7)
    ids = rng.integers(-2, 12, (20, 6))
    rows = MO.rows_of(ids, None, 10)
    count = np.zeros((20, 10))
    for r in range(20):
        for c in range(6):
            if 0 <= ids[r, c] < 10:
                count[r, ids[r, c]] += 1
    table, g = rng.standard_normal((10, 5)), rng.standard_normal((20, 5))
    np.testing.assert_allclose(MO.embed(table, rows, 0.5)[0], 0.5 * count @ table, atol=1e-12)
    np.testing.assert_allclose(MO.embed_backward(g, rows, 10, 0.5)[0], 0.5 * count.T @ g, atol=1e-12)
    assert MO.rows_of([[3, 3]], [0, 100], 50).tolist() == [[3, -1]]


# ---- the binding -------------------------------------------------------------------------------------


def test_binding_refuses_arrays_of_another_shape(api):
    import torch
    t = torch.zeros(6, 2)
    for bad in ((2, 6), (4, 3), (6, 1), 13):
        with pytest.raises(api.FsError):
            api._array(t, "w", bad, torch.float32)
    assert api._array(t, "w", (6, 2), torch.float32) == api._array(t, "w", 12, torch.float32) == t.data_ptr()
    assert api._array(t.view(-1), "w", (6, 2), torch.float32) == t.data_ptr()
    with pytest.raises(api.FsError):
        api._array(t.view(1, 12), "w", (6, 2), torch.float32)


def test_binding_refuses_numbers_that_32_bits_do_not_hold(api):
    """Not one of them reaches the library as its low 32 bits."""
    import torch
    for name in ("n_experts", "k", "score", "n_groups", "top_groups", "group_best"):
        with pytest.raises(api.FsError) as e:
            api.route_params(**{"n_experts": 8, "k": 2, name: (1 << 32) + 2})
        assert name in str(e.value)
    with pytest.raises(api.FsError):
        api._matrix(torch.empty(1, (1 << 32) + 8, device="meta"), "x")
    with pytest.raises(api.FsError):
        api._id_array(torch.empty(1, (1 << 32) + 1, device="meta", dtype=torch.int32), None)
    assert api._matrix(torch.empty(1, (1 << 31) - 1, device="meta"), "x")[1:] == (api.FS_F32, (1 << 31) - 1)


def test_binding_refuses_tensors_and_streams_of_a_gpu_that_is_not_the_current_one(api, monkeypatch):
    """Two GPUs as torch would report them."""
    import types

    import torch

    def tensor(index):
        return types.SimpleNamespace(is_cuda=True, device=torch.device("cuda", index))

    def stream(index):
        return types.SimpleNamespace(device_index=index, cuda_stream=77)

    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(api, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(api, "_gpus", 0, raising=False)
    assert api._Place(tensor(1), None).ptr == 101 and api._Place(tensor(1), stream(1)).ptr == 77
    for t, s in ((tensor(0), None), (tensor(0), stream(0)), (tensor(1), stream(0)), (tensor(0), stream(1))):
        with pytest.raises(api.FsError) as e:
            api._Place(t, s)
        assert "GPU" in str(e.value)
