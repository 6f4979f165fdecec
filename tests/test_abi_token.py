"""Host-side checks of the token losses' C entry points that need no GPU: bad arguments are
refused before anything is enqueued (these calls never reach the HIP runtime)."""
import ctypes
import os

import pytest

OK, INVALID, WORKSPACE = 0, 1, 2
F32, BF16, F16 = 0, 1, 2
P = ctypes.c_void_p(0x1000)     # never dereferenced: every call below fails its checks or is a no-op


@pytest.fixture(scope="module")
def lib():
    import paper_1911_05063_amd as cd
    if not os.path.exists(cd.LIB_PATH):
        from paper_1911_05063_amd import build
        build.build()
    return cd.library()


def score(lib, B=2, T=3, V=100, logits=P, dtype=F32, sb=300, st=100, tokens=P, temperature=1.0, top=0,
          logprob=P, entropy=P, top_logprob=P, top_token=P, saved=P, ws=P, ws_bytes=1 << 30):
    return lib.cd_token_logprobs_forward(B, T, V, logits, dtype, sb, st, tokens, temperature, top,
                                         logprob, entropy, top_logprob, top_token, saved, ws, ws_bytes,
                                         None)


def score_grad(lib, B=2, T=3, V=100, logits=P, saved=P, g=P, temperature=1.0, dtype=F32):
    return lib.cd_token_logprobs_backward(B, T, V, logits, dtype, 300, 100, P, temperature, saved, P, P,
                                          g, None)


def distill(lib, B=2, T=3, V=100, K=4, logits=P, dtype=F32, ids=P, t=P, tdtype=BF16, temperature=1.0,
            loss=P, saved=P, ws=P, ws_bytes=1 << 30):
    return lib.cd_distill_forward(B, T, V, K, logits, dtype, 300, 100, ids, t, tdtype, temperature, loss,
                                  saved, ws, ws_bytes, None)


def head(lib, B=2, T=3, D=64, V=100, h=P, w=P, dtype=BF16, sb=192, st=64, ld=64, tokens=P,
         temperature=1.0, logprob=P, entropy=P, saved=P, ws=P, ws_bytes=1 << 40):
    return lib.cd_head_logprobs_forward(B, T, D, V, h, w, dtype, sb, st, ld, tokens, temperature, logprob,
                                        entropy, saved, ws, ws_bytes, None)


def head_grad(lib, B=2, T=3, D=64, V=100, gh=P, gw=P, saved=P, ws=P, ws_bytes=1 << 40):
    return lib.cd_head_logprobs_backward(B, T, D, V, P, P, BF16, 192, 64, 64, P, 1.0, saved, P, P, gh, gw,
                                         ws, ws_bytes, None)


BAD_ROWS = [dict(B=-1), dict(T=-1), dict(V=0), dict(V=-5), dict(V=2 ** 31), dict(B=2 ** 16, T=2 ** 15),
            dict(B=2 ** 62, T=4), dict(dtype=3), dict(dtype=-1)]
BAD_TEMPERATURES = [0.0, -1.0, float("nan"), float("inf"), 1e-45]


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(sb=-1), dict(st=-1), dict(top=-1), dict(top=65),
                                            dict(V=10, top=11), dict(logits=None), dict(logprob=None),
                                            dict(entropy=None), dict(top=2, top_logprob=None),
                                            dict(top=2, top_token=None),
                                            dict(saved=ctypes.c_void_p(0x1004))])
def test_score_refuses(lib, bad):
    assert score(lib, **bad) == INVALID
    assert b"invalid argument" in lib.cd_last_error()


@pytest.mark.parametrize("t", BAD_TEMPERATURES)
def test_temperatures(lib, t):
    assert score(lib, temperature=t) == INVALID and score_grad(lib, temperature=t) == INVALID
    assert distill(lib, temperature=t) == INVALID and head(lib, temperature=t) == INVALID
    assert b"temperature" in lib.cd_last_error()


@pytest.mark.parametrize("t", [3e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_inverse_in_bits_overflows(lib, t):
    # 1 / t is finite, log2(e) / t is not: every difference of logits would be taken times infinity.
    test_temperatures(lib, t)


def test_distillation_squares_the_temperature(lib):
    assert distill(lib, temperature=1e30) == INVALID


@pytest.mark.parametrize("t", [1e-30, 1e-20])
def test_distillation_does_not_lose_the_squared_temperature(lib, t):
    # The loss would be 0 (or NaN where it is infinite) whatever the logits.
    assert distill(lib, temperature=t) == INVALID
    assert b"temperature^2" in lib.cd_last_error()
    assert distill(lib, temperature=t, loss=None) == INVALID
    assert distill(lib, temperature=2e-19, loss=None) == INVALID and b"NULL" in lib.cd_last_error()


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(K=0), dict(K=257), dict(logits=None), dict(ids=None),
                                            dict(t=None), dict(loss=None), dict(tdtype=7),
                                            dict(saved=ctypes.c_void_p(0x1008))])
def test_distill_refuses(lib, bad):
    assert distill(lib, **bad) == INVALID


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(D=0), dict(D=2 ** 21), dict(dtype=F32), dict(sb=-8),
                                            dict(st=-8), dict(ld=-8), dict(h=None), dict(w=None),
                                            dict(tokens=None), dict(logprob=None), dict(entropy=None),
                                            dict(h=ctypes.c_void_p(0x1002)), dict(w=ctypes.c_void_p(0x1008)),
                                            dict(saved=ctypes.c_void_p(0x1004)),
                                            dict(B=1, T=2 ** 30, V=2 ** 20)])
def test_head_refuses(lib, bad):
    assert head(lib, **bad) == INVALID


def test_backward_refuses(lib):
    for bad in (dict(logits=None), dict(saved=None), dict(g=None), dict(V=0), dict(dtype=5),
                dict(saved=ctypes.c_void_p(0x1001))):
        assert score_grad(lib, **bad) == INVALID
    assert head_grad(lib, saved=None) == INVALID
    assert head_grad(lib, gh=ctypes.c_void_p(0x1002)) == INVALID
    assert head_grad(lib, gw=ctypes.c_void_p(0x1008)) == INVALID
    assert head_grad(lib, ws=None) == WORKSPACE and head_grad(lib, ws_bytes=0) == WORKSPACE
    assert lib.cd_distill_backward(2, 3, 100, 4, P, F32, 300, 100, P, P, F32, 1.0, P, None, P,
                                   None) == INVALID


def test_no_rows_is_a_no_op(lib):
    none = dict(logits=None, logprob=None, entropy=None, ws=None, ws_bytes=0)
    assert score(lib, B=0, **none) == OK and score(lib, T=0, **none) == OK
    assert score_grad(lib, B=0, logits=None, saved=None, g=None) == OK
    assert distill(lib, T=0, logits=None, ids=None, t=None, loss=None, ws=None) == OK
    assert head(lib, T=0, h=None, w=None, tokens=None, ws=None, ws_bytes=0) == OK
    assert head_grad(lib, B=0, saved=None, ws=None) == OK
    assert head_grad(lib, gh=None, gw=None, saved=None, ws=None) == OK


def test_workspaces(lib):
    # Rows are cut over workgroups, and need a workspace, only where few and very long.
    assert lib.cd_token_workspace_bytes(1, 4096, 65536, BF16, 64) == 0
    need = lib.cd_token_workspace_bytes(1, 1, 1 << 20, F32, 20)
    assert need > 0 and need % 256 == 0
    assert score(lib, B=1, T=1, V=1 << 20, top=20, ws_bytes=need - 1) == WORKSPACE
    assert b"workspace too small" in lib.cd_last_error()
    assert score(lib, B=1, T=1, V=1 << 20, top=20, ws=None) == WORKSPACE
    assert score(lib, B=1, T=1, V=1 << 20, top=20, ws=ctypes.c_void_p(0x1010)) == INVALID
    assert distill(lib, B=1, T=1, V=1 << 20, ws_bytes=1) == WORKSPACE
    for bad in ((-1, 1, 10, F32, 0), (1, 1, 0, F32, 0), (1, 1, 10, 4, 0), (1, 1, 10, F32, 11),
                (1, 1, 100, F32, 65), (0, 5, 10, F32, 0)):
        assert lib.cd_token_workspace_bytes(*bad) == 0

    def h(T, D, V, backward, ld=None, st=None):
        return lib.cd_head_workspace_bytes(1, T, D, V, BF16, 0, D if st is None else st,
                                           D if ld is None else ld, backward)
    assert h(0, 64, 100, 0) == 0 and h(4, 0, 100, 0) == 0
    need = h(6, 64, 100, 0)
    assert head(lib, B=1, T=6, sb=0, ws_bytes=need - 1) == WORKSPACE
    assert head(lib, B=1, T=6, sb=0, ws=None) == WORKSPACE
    assert head(lib, B=1, T=6, sb=0, ws=ctypes.c_void_p(0x1010)) == INVALID
    # Copies of hidden and weight only where they cannot be read in place.
    assert h(1000, 64, 5000, 0) < h(1000, 60, 5000, 0)              # hidden: D is no multiple of 64
    assert h(1000, 72, 50000, 0) + 50000 * 72 * 2 <= h(1000, 70, 50000, 0)      # weight: none of 8
    assert h(1000, 64, 5000, 0, st=68) > h(1000, 64, 5000, 0, st=72)
    # The backward never holds all of d/d logits of a large problem.
    assert h(8192, 2048, 200000, 1) < 1 << 30
    assert 8192 * 200000 * 2 > 3 << 30
