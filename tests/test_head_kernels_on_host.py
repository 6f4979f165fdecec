"""The kernels of head_loss.hip and the matrix product of tile_product.h, compiled for the CPU
(host_lanes/lanes.h), on buffers that end or begin at an unmapped page: every access is inside them,
the results are the oracle's, and they do not depend on when loads to LDS arrive between being asked for
and being waited for, nor on the order of the waves between barriers."""
import ctypes
import os

import numpy as np
import pytest

import host_kernels
from host_kernels import BF16, F16, in_child, place, ptr, stored, values
from oracle import token_oracle as o


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not os.path.exists(host_kernels.CLANG):
        pytest.skip("no clang++ of ROCm")
    return ctypes.CDLL(host_kernels.build(str(tmp_path_factory.mktemp("host_lanes")), "head",
                                          os.path.join(host_kernels.CSRC, "head_loss.hip")))


def aligned(a, at_end):
    """place(), 16-byte aligned (its end is at most 14 bytes before the unmapped page)."""
    pad = -a.nbytes % 16 // a.itemsize
    return place(np.concatenate([a.reshape(-1), np.zeros(pad, a.dtype)]), at_end)


def run(lib, B, T, D, V, dtype, gap, at_end, early, backwards, grads=True):
    lib.host_order(early, backwards)
    rng = np.random.default_rng(B + 7 * T + 31 * D + 101 * V)
    R = B * T
    h, hv = stored(rng.normal(size=(R, D)), dtype)
    w, wv = stored(rng.normal(size=(V, D)) * 3 / np.sqrt(D), dtype)
    ld = D + gap
    wide = np.full((V, ld), 0x7FFF if dtype == BF16 else np.nan).astype(w.dtype)    # NaN
    wide[:, :D] = w
    tokens = rng.integers(0, V, R).astype(np.int32)
    if R > 2:
        tokens[0], tokens[1], tokens[2] = V - 1, V, -1
    i64, temperature, f32 = ctypes.c_int64, ctypes.c_float(1.5), np.float32
    hidden, weight = aligned(h, at_end), aligned(wide.reshape(-1)[:(V - 1) * ld + D], at_end)
    tokens = place(tokens, at_end)
    sizes = [i64(B), i64(T), i64(D), i64(V), i64(T * D), i64(D), i64(ld), dtype]
    lp, ent = (place(np.full(R, 7, f32), at_end) for _ in range(2))
    saved = place(np.zeros((R, 4), f32), at_end)
    lib.host_head_workspace.restype = ctypes.c_size_t

    def workspace(backward):       # full of NaN: nothing of it is used that the call did not write
        return place(np.full(lib.host_head_workspace(*sizes, backward), 0xFF, np.uint8), at_end)

    lib.host_head(ptr(hidden), ptr(weight), *sizes, ptr(tokens), temperature, ptr(lp), ptr(ent), ptr(saved),
                  ptr(workspace(0)))
    rl, re = o.head_logprobs(hv, wv, tokens, 1.5)
    np.testing.assert_allclose(lp, rl, rtol=1e-5, atol=1e-4)
    np.testing.assert_allclose(ent, re, rtol=1e-5, atol=1e-4)
    if not grads:
        return
    gl, ge = (place(rng.normal(size=R).astype(f32), at_end) for _ in range(2))
    gh, gw = (aligned(np.full(n, 7, h.dtype), at_end) for n in (R * D, V * D))
    lib.host_head_grad(ptr(hidden), ptr(weight), *sizes, ptr(tokens), temperature, ptr(saved), ptr(gl), ptr(ge),
                       ptr(gh), ptr(gw), ptr(workspace(1)))
    rh, rw = o.head_logprobs_grad(hv, wv, tokens, gl, ge, 1.5)
    # d/d logits and the results are rounded to the type: 2 roundings of each term's size.
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -11
    dx = np.abs(o.token_logprobs_grad(hv @ wv.T, tokens, gl, ge, 1.5))
    for got, ref, size in ((gh, rh, dx @ np.abs(wv)), (gw, rw, dx.T @ np.abs(hv))):
        got = values(got, dtype)[:ref.size].reshape(ref.shape)
        assert np.all(np.abs(got - ref) <= u * (np.abs(ref) + 2 * size) + 1e-5)


# (T, D, V): D of whole steps of 64 or not, of whole 16 bytes or not; few rows, and parts of
# a sum.
SHAPES = [(1, 1, 1, 1, BF16, 0), (1, 3, 7, 5, F16, 0), (1, 5, 72, 300, BF16, 0), (1, 5, 72, 300, BF16, 16),
          (2, 9, 64, 130, F16, 0), (1, 130, 200, 140, BF16, 8), (1, 17, 320, 270, F16, 64), (1, 300, 40, 129, BF16, 8),
          (1, 257, 1100, 30, BF16, 0), (1, 40, 8, 1300, F16, 8)]


@pytest.mark.parametrize("at_end,early,backwards", [(True, 0, 0), (False, 1, 1), (True, 1, 0), (True, 0, 1)])
@pytest.mark.parametrize("B,T,D,V,dtype,gap", SHAPES)
def test_head(lib, B, T, D, V, dtype, gap, at_end, early, backwards):
    in_child(run, lib, B, T, D, V, dtype, gap, at_end, early, backwards)


@pytest.mark.slow
@pytest.mark.parametrize("T,D,V,early,backwards", [(300, 8, 20400, 0, 0), (5, 300, 20400, 0, 1),
                                                   (20400, 300, 5, 1, 0)])
def test_tiles_of_256(lib, T, D, V, early, backwards):
    # In turn: logits (some workgroups take one tile, in 160 in all) and d/d logits, d/d weights, d/d hidden.
    in_child(run, lib, 1, T, D, V, BF16, 8 if D % 8 == 0 else 0, True, early, backwards)


def test_scale_of_many_rows(lib):
    # Several workgroups look for the scale of float16 gradients.
    in_child(run, lib, 1, 9000, 8, 20, F16, 0, True, 0, 0)
