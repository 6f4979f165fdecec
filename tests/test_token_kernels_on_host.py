"""The kernels of token_loss.hip, compiled for the CPU (host_lanes/lanes.h), on buffers that end or
begin at an unmapped page: every access is inside them for the ways a row is shared out (16 lanes, a
wave, 4 and 16 waves, cuts), odd row lengths, repeated entries and rows of few values, and the results
are the oracle's."""
import ctypes
import faulthandler
import multiprocessing
import os

import numpy as np
import pytest

import host_kernels
from host_kernels import BF16, F16, F32, in_child, place, ptr, stored, values
from oracle import token_oracle as o


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not os.path.exists(host_kernels.CLANG):
        pytest.skip("no clang++ of ROCm")
    return ctypes.CDLL(host_kernels.build(str(tmp_path_factory.mktemp("host_lanes")), "token",
                                          os.path.join(host_kernels.CSRC, "token_loss.hip")))


# Tolerances: a sum of V weights in float32 and its statistics, as on the GPU (far below 1e-4 for
# log-probabilities of size 30); gradients as rounded to their type.
ROUND = {F32: 1e-6, BF16: 2.0 ** -8, F16: 2.0 ** -11}


def run_score(lib, B, T, V, dtype, top, kind, at_end, gap=0):
    rng = np.random.default_rng(B + 7 * T + 31 * V + top)
    R = B * T
    x = rng.normal(size=(R, V)) * 3
    if kind == "masked":
        x[rng.random((R, V)) < 0.5] = -np.inf
        x[0] = -np.inf
    elif kind == "equal":
        x[:] = rng.integers(0, 2, (R, 1))
    elif kind == "descending":
        x = -np.tile(np.arange(V) / 64.0, (R, 1))
    raw, xv = stored(x, dtype)
    rows = np.zeros((R, V + gap), raw.dtype)
    rows[:, :V] = raw
    held = place(rows.reshape(-1)[:(R - 1) * (V + gap) + V], at_end)    # ends with the last row
    tokens = rng.integers(0, V, R).astype(np.int32)
    if R > 2:
        tokens[1], tokens[2] = -1, V
    tokens = place(tokens, at_end)
    f = lambda *s: place(np.full(s, 7, np.float32), at_end)     # noqa: E731
    lp, ent = f(R), f(R)
    tlp, tt = (f(R, top), place(np.full((R, top), 7, np.int32), at_end)) if top else (None, None)
    saved = place(np.zeros((R, 4), np.float32), at_end)
    lib.host_workspace.restype = ctypes.c_size_t
    ws = place(np.zeros(lib.host_workspace(ctypes.c_int64(R), ctypes.c_int64(V), dtype, top), np.uint8), at_end)
    i64, temperature = ctypes.c_int64, ctypes.c_float(1.3)
    sizes = [i64(B), i64(T), i64(V), i64(T * (V + gap)), i64(V + gap), dtype]
    lib.host_score(ptr(held), *sizes, ptr(tokens), temperature, top, ptr(lp), ptr(ent), ptr(tlp), ptr(tt),
                   ptr(saved), ptr(ws))
    ref = o.token_logprobs(xv, tokens, top, np.float32(1.3).astype(np.float64))
    close = lambda a, b, t: np.testing.assert_allclose(a, b, rtol=1e-5, atol=t)     # noqa: E731
    close(lp, ref["logprob"], 1e-4)
    close(ent, ref["entropy"], 1e-4)
    if top:
        assert np.array_equal(tt, ref["top_token"])
        close(tlp, ref["top_logprob"], 1e-4)
        return
    gl, ge = f(R), f(R)
    gl[:], ge[:] = rng.normal(size=R), rng.normal(size=R)
    gx = place(np.full((R, V), 7, raw.dtype), at_end)
    lib.host_score_grad(ptr(held), *sizes, ptr(tokens), temperature, ptr(saved), ptr(gl), ptr(ge), ptr(gx))
    np.testing.assert_allclose(values(gx, dtype), o.token_logprobs_grad(xv, tokens, gl, ge, 1.3),
                               rtol=1.1 * ROUND[dtype] + 1e-4, atol=1e-5)


def run_distill(lib, R, V, K, dtype, teacher_dtype, repeat, at_end):
    rng = np.random.default_rng(R + 7 * V + 31 * K)
    raw, xv = stored(rng.normal(size=(R, V)) * 3, dtype)
    ids = np.stack([rng.permutation(max(V, K))[:K] for _ in range(R)])
    if repeat:
        ids = rng.integers(0, max(1, V // 3), (R, K))
    ids = np.where((ids < V) & (rng.random((R, K)) > 0.1), ids, -1).astype(np.int32)
    if R > 2:
        ids[1] = -1
        ids[2, 0] = V
    ids[0, 0] = V - 1
    traw, tv = stored(rng.normal(size=(R, K)) * 2, teacher_dtype)
    held, ids, traw = place(raw, at_end), place(ids, at_end), place(traw, at_end)
    loss = place(np.full(R, 7, np.float32), at_end)
    saved = place(np.zeros((R, 8), np.float32), at_end)
    lib.host_workspace.restype = ctypes.c_size_t
    ws = place(np.zeros(lib.host_workspace(ctypes.c_int64(R), ctypes.c_int64(V), dtype, 0), np.uint8), at_end)
    i64, temperature = ctypes.c_int64, ctypes.c_float(1.5)
    sizes = [i64(1), i64(R), i64(V), i64(0), i64(V), dtype, K]
    lib.host_distill(ptr(held), *sizes, ptr(ids), ptr(traw), teacher_dtype, temperature, ptr(loss), ptr(saved),
                     ptr(ws))
    np.testing.assert_allclose(loss, o.distill(xv, ids, tv, 1.5), rtol=1e-4, atol=1e-4)
    g = place(rng.normal(size=R).astype(np.float32), at_end)
    gx = place(np.full((R, V), 7, raw.dtype), at_end)
    lib.host_distill_grad(ptr(held), *sizes, ptr(ids), ptr(traw), teacher_dtype, temperature, ptr(saved), ptr(g),
                          ptr(gx))
    np.testing.assert_allclose(values(gx, dtype), o.distill_grad(xv, ids, tv, g, 1.5),
                               rtol=1.1 * ROUND[dtype] + 1e-4, atol=1e-5)


@pytest.mark.parametrize("at_end", [True, False])
@pytest.mark.parametrize("B,T,V,dtype,kind", [
    (1, 3, 1, BF16, ""), (2, 3, 7, F16, ""), (1, 5, 9, BF16, ""), (1, 33, 1023, BF16, "masked"),
    (3, 4, 511, F32, ""), (1, 3, 2051, F16, ""), (1, 2, 5003, F32, "masked"), (1, 600, 1100, BF16, ""),
    (1, 3, 16385, BF16, ""), (1, 2, 70001, BF16, ""), (1, 2, 8197, F32, ""), (1, 1, 262201, BF16, "")])
def test_scores_and_gradients(lib, B, T, V, dtype, kind, at_end):
    in_child(run_score, lib, B, T, V, dtype, 0, kind, at_end, 3)


@pytest.mark.parametrize("at_end", [True, False])
@pytest.mark.parametrize("T,V,dtype,top,kind", [
    (3, 1, BF16, 1, ""), (5, 7, F32, 7, ""), (5, 70, F16, 64, "equal"), (600, 130, BF16, 5, ""),
    (3, 2051, F32, 64, "masked"), (3, 4104, BF16, 20, ""), (1, 9001, BF16, 64, "descending"),
    (3, 70001, BF16, 64, ""), (3, 70001, BF16, 64, "equal"), (1, 70001, F16, 64, "masked"),
    (1, 70003, BF16, 33, "descending"), (2, 16391, BF16, 64, ""), (2, 9001, F32, 64, "equal"),
    (1, 262201, BF16, 64, ""), (1, 262201, BF16, 64, "masked"), (1, 140001, F32, 20, "")])
def test_alternatives(lib, T, V, dtype, top, kind, at_end):
    in_child(run_score, lib, 1, T, V, dtype, top, kind, at_end, 1)


@pytest.mark.parametrize("at_end", [True, False])
@pytest.mark.parametrize("R,V,K,dtype,teacher,repeat", [
    (1, 1, 1, BF16, BF16, False), (5, 7, 3, F32, F16, False), (33, 64, 64, BF16, F32, True),
    (7, 1000, 256, F16, F16, True), (3, 2051, 129, F32, BF16, False), (3, 2051, 256, BF16, BF16, True),
    (2, 20001, 64, BF16, F32, True), (1, 262201, 256, BF16, BF16, True)])
def test_distillation(lib, R, V, K, dtype, teacher, repeat, at_end):
    in_child(run_distill, lib, R, V, K, dtype, teacher, repeat, at_end)


def test_an_access_outside_a_buffer_is_seen(lib):
    # A row shorter than the kernel is told (planted here, on the host): the harness notices.
    def planted():
        real = globals()["place"]
        faulthandler.disable()
        globals()["place"] = lambda a, at_end: real(a[:-1] if a.ndim == 1 and a.size > 70000 else a, at_end)
        run_score(lib, 1, 1, 70001, BF16, 64, "", True)
    p = multiprocessing.get_context("fork").Process(target=planted)
    p.start()
    p.join()
    assert p.exitcode < 0
