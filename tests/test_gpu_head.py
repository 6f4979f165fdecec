"""Log-probabilities from hidden states and the vocabulary matrix on the GPU against the
float64 oracle, with the gradients to both."""
import numpy as np
import pytest
import torch

import paper_1911_05063_amd as cd
from oracle import token_oracle as o

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}     # unit roundoff
EPS = 2.0 ** -24


def n64(t):
    return t.detach().double().cpu().numpy()


def make(rng, T, D, V, dtype, spread=3.0):
    h = torch.from_numpy(rng.normal(size=(T, D))).to(DTYPES[dtype]).cuda()
    w = torch.from_numpy(rng.normal(size=(V, D)) * spread / np.sqrt(D)).to(DTYPES[dtype]).cuda()
    tokens = rng.integers(0, V, T).astype(np.int32)
    tokens[rng.random(T) < 0.15] = -1
    return h, w, tokens


# Tolerances.  A logit is a sum of D products, exact in float32 each, in a chain of D / 32
# accumulations of 32: its error is below EPS (D / 32 + 32) sum |h w|, and typically a
# fraction; x_err below takes the whole bound.  log p and the entropy (whose derivative by a logit is
# at most 1 + log V) inherit it, with the softmax's own error.
def x_error(h, w, T):
    return EPS * (h.shape[1] / 32 + 32) * (np.abs(h) @ np.abs(w).T).max() / T + EPS * 80


def check(h, w, tokens, dtype, T=1.0, gscale=1.0, grads=True, hv=None):
    """hv: the view of h that is handed over, if not h itself."""
    rng = np.random.default_rng(5)
    V = w.shape[0]
    hg = (h if hv is None else hv).detach().requires_grad_(grads)
    wg = w.detach().requires_grad_(grads)
    tg = torch.from_numpy(tokens).cuda().view(hg.shape[:-1])
    lp, ent = cd.head_logprobs(hg, wg, tg, temperature=T)
    hn, wn = n64(hg).reshape(-1, w.shape[1]), n64(w)
    rl, re = o.head_logprobs(hn, wn, tokens, T)
    e = x_error(hn, wn, T)
    got_l, got_e = n64(lp).reshape(-1), n64(ent).reshape(-1)
    assert np.all((np.abs(got_l - rl) <= 2 * e + 4 * EPS * np.abs(rl)) | (np.isnan(got_l) & np.isnan(rl)))
    assert np.all(np.abs(got_e - re) <= e * (2 + 2 * np.log(V + 1)))
    if not grads:
        return lp, ent
    gl = (rng.normal(size=len(rl)) * gscale).astype(np.float32)
    ge = (rng.normal(size=len(rl)) * gscale * 0.1).astype(np.float32)
    gh, gw = torch.autograd.grad([lp, ent], [hg, wg], [torch.from_numpy(g).cuda().view(lp.shape)
                                                       for g in (gl, ge)])
    assert gh.shape == hg.shape and gh.dtype == hg.dtype and gw.shape == w.shape and gw.dtype == w.dtype
    rh, rw = o.head_logprobs_grad(hn, wn, tokens, gl, ge, T)
    # dx is rounded once (UNIT of it) and carries the logits' error; both add up over the
    # products' terms; the sums of float32 products add EPS per step, the result UNIT.
    dx = np.abs(o.token_logprobs_grad(hn @ wn.T, tokens, gl, ge, T))
    p = np.exp(o._log_softmax(hn @ wn.T / T))
    live = (tokens >= 0)[:, None]
    size = live * p * (np.abs(gl) + np.abs(ge) * (2 * np.log(V + 1) + 4))[:, None] / T
    err = UNIT[dtype] * dx + size * 4 * e
    if dtype == "f16":      # what lies below float16's normal numbers: 2^-25 of the scaled element
        err = err + 2.0 ** -38 * (np.abs(gl).max() + np.abs(ge).max() * (np.log(V) + 1)) / T * live
    chain = lambda n: EPS * (n / 32 + 64)  # noqa: E731
    u, tiny = UNIT[dtype], (2.0 ** -24 if dtype == "f16" else 1e-37)
    tol_h = err @ np.abs(wn) + chain(V) * (dx @ np.abs(wn)) + 1.01 * u * np.abs(rh) + tiny
    tol_w = err.T @ np.abs(hn) + chain(len(rl)) * (dx.T @ np.abs(hn)) + 1.01 * u * np.abs(rw) + tiny
    for got, ref, tol in ((gh, rh, tol_h), (gw, rw, tol_w)):
        bad = np.abs(n64(got).reshape(ref.shape) - ref) > tol
        assert not bad.any(), (np.argwhere(bad)[:4], n64(got).reshape(ref.shape)[bad][:4], ref[bad][:4])
    return lp, ent


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,D,V", [(1, 1, 1), (1, 64, 300), (2, 7, 5), (16, 64, 128), (17, 200, 1000),
                                   (129, 100, 257), (300, 64, 129), (255, 72, 513), (64, 1000, 130),
                                   (1030, 192, 700), (2, 130, 5000)])
def test_logprobs_and_gradients(T, D, V, dtype):
    rng = np.random.default_rng(T + 31 * D + 1009 * V)
    h, w, tokens = make(rng, T, D, V, dtype)
    if T > 2:
        tokens[0], tokens[1] = V - 1, V
    check(h, w, tokens, dtype, [1.0, 0.7, 2.0][T % 3], 1.0 if dtype == "bf16" else 300.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("D,V", [(8, 33), (136, 700), (1096, 95), (2056, 320)])
def test_few_rows(T, D, V, dtype):
    rng = np.random.default_rng(T + 31 * D + 1009 * V)
    h, w, tokens = make(rng, T, D, V, dtype)
    if T > 1:
        tokens[0], tokens[1] = V - 1, V
    check(h, w, tokens, dtype, [1.0, 0.7, 2.0][T % 3], 1.0 if dtype == "bf16" else 300.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_tiles(dtype):
    # 13 x 13 tiles of 256 forward, the same of d/d logits; D is no multiple of 64.
    rng = np.random.default_rng(11)
    h, w, tokens = make(rng, 3200, 40, 3300, dtype)
    check(h, w, tokens, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_workgroups_that_take_several_tiles(dtype):
    # 17 x 36 tiles of 256 on 256 workgroups, the last of both sides cut off.
    rng = np.random.default_rng(13)
    h, w, tokens = make(rng, 4200, 72, 9100, dtype)
    tokens[::7] = -1
    tokens[-1], tokens[-2] = 9099, 9100
    check(h, w, tokens, dtype)


@pytest.mark.parametrize("T,D,V", [(3300, 3200, 300), (200, 3200, 3300)])
def test_large_tiles_of_the_gradients(T, D, V):
    rng = np.random.default_rng(12)
    h, w, tokens = make(rng, T, D, V, "bf16")
    check(h, w, tokens, "bf16")


def test_small_float16_gradients_do_not_vanish():
    # p / 4096 is below float16's smallest number for most of the vocabulary.
    rng = np.random.default_rng(13)
    h, w, tokens = make(rng, 40, 64, 2000, "f16")
    check(h, w, tokens, "f16", gscale=2.0 ** -12)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 3, 40, 256])
def test_gradients_of_few_rows_are_rounded_once(T, dtype):
    # d/d logits is held in two parts, together at most UNIT^2 off: what is left is the
    # result's own rounding, the logits' error (in p, x_error) and the sums' (EPS a step).
    rng = np.random.default_rng(19 + T)
    h, w, tokens = make(rng, T, 128, 1200, dtype)
    tokens = np.abs(tokens)
    hg, wg = h.requires_grad_(), w.requires_grad_()
    lp, _ = cd.head_logprobs(hg, wg, torch.from_numpy(tokens).cuda())
    g = rng.normal(size=T).astype(np.float32)
    gh, gw = torch.autograd.grad([lp], [hg, wg], [torch.from_numpy(g).cuda()])
    hn, wn = n64(h), n64(w)
    x = hn @ wn.T
    dx = o.token_logprobs_grad(x, tokens, g, np.zeros(T))
    err = np.exp(o._log_softmax(x)) * np.abs(g)[:, None] * 2 * x_error(hn, wn, 1.0)
    err = err + np.abs(dx) * (UNIT[dtype] ** 2 + EPS * (1200 / 32 + 64))
    if dtype == "f16":      # below float16's normal numbers, of the scaled element
        err = err + 2.0 ** -38 * np.abs(g).max()
    tiny = 2.0 ** -24 if dtype == "f16" else 1e-37
    for got, ref, e in ((gh, dx @ wn, err @ np.abs(wn)), (gw, dx.T @ hn, err.T @ np.abs(hn))):
        assert np.all(np.abs(n64(got) - ref) <= 1.001 * UNIT[dtype] * np.abs(ref) + e + tiny)


def test_hidden_is_read_in_place_or_copied():
    rng = np.random.default_rng(14)
    for D in (64, 72, 51):
        big = torch.from_numpy(rng.normal(size=(5, 9, 200))).bfloat16().cuda()
        w = torch.from_numpy(rng.normal(size=(333, 200)) / 4).bfloat16().cuda()
        for off in (0, 8, 3):
            for view in (big[:, :-1, off:off + D], big[2, :, off:off + D], big[:, ::2, off:off + D],
                         big.transpose(0, 1)[..., off:off + D], big[0, 0, off:off + D].expand(6, D),
                         big[0, 0, off:off + D]):
                n = view.numel() // D
                tokens = rng.integers(0, 333, n).astype(np.int32)
                check(None, w[:, off:off + D], tokens, "bf16", hv=view)


def test_rows_without_a_token_may_hold_anything():
    rng = np.random.default_rng(15)
    h, w, tokens = make(rng, 70, 64, 500, "bf16")
    none = tokens < 0
    assert none.any()
    clean = check(h, w, tokens, "bf16")
    hg, wg = h.clone(), w.clone().requires_grad_()
    hg[torch.from_numpy(none).cuda()] = float("nan")
    hg.requires_grad_()
    tg = torch.from_numpy(tokens).cuda()
    lp, ent = cd.head_logprobs(hg, wg, tg)
    gh, gw = torch.autograd.grad(lp.sum() + ent.sum(), [hg, wg])
    assert torch.equal(lp, clean[0]) and torch.equal(ent, clean[1])
    assert torch.isfinite(gw).all() and not gh[torch.from_numpy(none).cuda()].any()
    # All rows unused: zeros.
    lp, ent = cd.head_logprobs(hg, wg, torch.full_like(tg, -1))
    gh, gw = torch.autograd.grad(lp.sum() + ent.sum(), [hg, wg])
    assert not lp.any() and not ent.any() and not gh.any() and not gw.any()


def test_nan_stays_in_its_row():
    rng = np.random.default_rng(16)
    h, w, tokens = make(rng, 20, 64, 300, "bf16")
    tokens[:] = 7
    h[3, 5] = float("nan")
    lp, ent = cd.head_logprobs(h, w, torch.from_numpy(tokens).cuda())
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[3] = True
    assert torch.equal(lp.isnan(), bad) and torch.equal(ent.isnan(), bad)


def test_ranges_of_the_vocabulary():
    # So many rows take ranges of 1024 columns of d/d logits: three here, the last short.
    rng = np.random.default_rng(17)
    T, D, V = 300000, 16, 2100
    h = torch.randn(T, D, device="cuda").bfloat16().requires_grad_()
    w = torch.randn(V, D, device="cuda").bfloat16().requires_grad_()
    tokens = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32)
    lp, ent = cd.head_logprobs(h, w, tokens)
    g0 = torch.rand(T, device="cuda")
    gh, gw = torch.autograd.grad([lp], [h, w], [g0])
    x = (h.detach().float() @ w.detach().float().t())
    used = tokens >= 0
    want = torch.log_softmax(x, 1)
    ref = torch.where(used, want.gather(1, tokens.clamp_min(0).long()[:, None])[:, 0], 0)
    assert (lp - ref).abs().max() < 1e-4
    d = -want.exp_() * (g0 * used)[:, None]
    d.scatter_add_(1, tokens.clamp_min(0).long()[:, None], (g0 * used)[:, None])
    rh, rw = d @ w.detach().float(), d.t() @ h.detach().float()
    # dx and the result rounded to 2^-8 each.
    sh = d.abs() @ w.detach().float().abs()
    sw = d.abs().t() @ h.detach().float().abs()
    assert ((gh.float() - rh).abs() <= 2.0 ** -7 * sh + 1e-6).all()
    assert ((gw.float() - rw).abs() <= 2.0 ** -7 * sw + 1e-6).all()


def test_only_the_wanted_gradients_and_the_same_bits():
    rng = np.random.default_rng(18)
    h, w, tokens = make(rng, 500, 128, 1500, "bf16")
    tg = torch.from_numpy(tokens).cuda()

    def grads(hr, wr):
        a, b = h.detach().requires_grad_(hr), w.detach().requires_grad_(wr)
        lp, ent = cd.head_logprobs(a, b, tg)
        wanted = [t for t in (a, b) if t.requires_grad]
        return torch.autograd.grad(lp.sum() - ent.sum(), wanted)

    both = grads(True, True)
    assert torch.equal(grads(True, False)[0], both[0]) and torch.equal(grads(False, True)[0], both[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = grads(True, True)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(both, again))


def test_no_rows():
    h = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    w = torch.randn(10, 64, device="cuda").bfloat16().requires_grad_()
    lp, ent = cd.head_logprobs(h, w, torch.empty(0, dtype=torch.int32, device="cuda"))
    gh, gw = torch.autograd.grad(lp.sum() + ent.sum(), [h, w])
    assert lp.shape == (0,) and gh.shape == h.shape and not gw.any()


def test_refusals():
    h = torch.randn(4, 64, device="cuda").bfloat16()
    w = torch.randn(100, 64, device="cuda").bfloat16()
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad, err in [((h.float(), w.float(), t), TypeError), ((h, w.half(), t), TypeError),
                     ((h, w, t.long()), TypeError), ((h, w, t[:3]), ValueError),
                     ((h, w[:, :32], t), ValueError), ((h.cpu(), w, t), ValueError),
                     ((h, w.cpu(), t), ValueError), ((h, w[:0], t), ValueError), ((h, w[0], t), ValueError),
                     ((h, None, t), TypeError), ((h, w, None), TypeError),
                     ((h[:, :0], w[:, :0], t), ValueError)]:
        with pytest.raises(err):
            cd.head_logprobs(*bad)
    for temperature in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(cd.CDError):
            cd.head_logprobs(h, w, t, temperature=temperature)


@pytest.mark.parametrize("around", [float("nan"), float("inf"), 1e30])
@pytest.mark.parametrize("T,D,V,ld", [(5, 72, 700, 200), (40, 8, 333, 16), (300, 1000, 333, 1024),
                                      (129, 40, 257, 48), (3200, 40, 3300, 48)])
def test_what_lies_between_the_rows_of_the_weights_is_not_used(T, D, V, ld, around):
    # Rows of a multiple of 8, not of 64, and further apart than they are long.
    rng = np.random.default_rng(T + D)
    h, w, tokens = make(rng, T, D, V, "bf16")
    wide = torch.full((V, ld), around, device="cuda").bfloat16()
    for off in (0, 8):
        if off + D <= ld:
            wide[:] = around
            wide[:, off:off + D] = w
            got = check(h, wide[:, off:off + D], tokens, "bf16", grads=T < 1000)
            # The same bits as of weights without a gap.
            hg, wg, tg = h.clone().requires_grad_(), w.clone().requires_grad_(), torch.from_numpy(tokens).cuda()
            lp, ent = cd.head_logprobs(hg, wg, tg)
            assert torch.equal(lp, got[0]) and torch.equal(ent, got[1])
            one = torch.ones_like(lp)
            want = torch.autograd.grad([lp, ent], [hg, wg], [one, one])
            view = wide[:, off:off + D].detach().requires_grad_()
            some = torch.autograd.grad(cd.head_logprobs(hg, view, tg), [hg, view], [one, one])
            assert all(torch.equal(a, b) for a, b in zip(some, want))


@pytest.mark.parametrize("T", [40, 300, 9001])
@pytest.mark.parametrize("big", [1e6, 1e30, float("inf"), float("nan")])
def test_float16_gradients_of_rows_that_take_none_do_not_scale_the_others(T, big):
    rng = np.random.default_rng(21)
    h, w, tokens = make(rng, T, 64, 2000, "f16")
    tokens[3], tokens[5] = -1, 2000             # no token; one past the vocabulary
    tg = torch.from_numpy(tokens).cuda()
    none, past = tg < 0, tg >= 2000

    def grads(gl, ge):
        a, b = h.clone().requires_grad_(), w.clone().requires_grad_()
        return torch.autograd.grad(cd.head_logprobs(a, b, tg), [a, b], [gl, ge])

    gl = torch.from_numpy(rng.normal(size=T).astype(np.float32)).cuda() * 2.0 ** -13
    ge = gl.flip(0) * 0.1
    clean = torch.where(none | past, 0.0, gl), torch.where(none, 0.0, ge)
    want = grads(*clean)
    assert want[0].any() and want[1].any()
    got = grads(torch.where(none | past, big, gl), torch.where(none, big, ge))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("big", [float("inf"), float("nan")])
def test_a_float16_gradient_that_is_not_finite_stays_in_its_row(big):
    rng = np.random.default_rng(22)
    h, w, tokens = make(rng, 40, 64, 2000, "f16")
    tokens = np.abs(tokens)
    tg = torch.from_numpy(tokens).cuda()

    def grad(gl):
        a = h.clone().requires_grad_()
        return torch.autograd.grad(cd.head_logprobs(a, w, tg)[0], a, gl)[0]

    gl = torch.from_numpy(rng.normal(size=40).astype(np.float32)).cuda() * 2.0 ** -13
    gl[11] = 0.0
    want = grad(gl)
    gl[11] = big
    got = grad(gl)
    rest = torch.arange(40, device="cuda") != 11
    assert torch.equal(got[rest], want[rest]) and not torch.isfinite(got[11]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 16, 33, 128])
@pytest.mark.parametrize("D,V", [(64, 700), (192, 1000), (1088, 400), (2048, 320)])
def test_few_rows_whose_workgroups_start_at_different_k(T, D, V, dtype):
    # One row of tiles, D a multiple of 64: of 1, 3, 17 and 32 steps of k each of the (up to 8)
    # tiles of the vocabulary begins at another and goes round.
    rng = np.random.default_rng(T + 31 * D + 1009 * V)
    h, w, tokens = make(rng, T, D, V, dtype)
    if T > 1:
        tokens[0], tokens[1] = V - 1, V
    check(h, w, tokens, dtype, [1.0, 0.7, 2.0][T % 3], 1.0 if dtype == "bf16" else 300.0)


@pytest.mark.parametrize("T,dtype", [(3, "bf16"), (70, "f16")])
def test_few_rows_of_weights_that_go_past_the_caches(T, dtype):
    rng = np.random.default_rng(23)
    D, V = 1024, 65537                          # more than 128 MB, the last tile of one column
    h, w, tokens = make(rng, T, D, V, dtype)
    tokens[0], tokens[1], tokens[2] = V - 1, V, -1
    check(h, w, tokens, dtype, gscale=1.0 if dtype == "bf16" else 300.0)


def test_ranges_of_the_vocabulary_over_few_rows():
    # d/d logits in two parts, and two ranges of 524288 columns, the last short.
    T, D, V = 200, 16, 600001
    g = torch.Generator(device="cuda").manual_seed(24)
    h = torch.randn(T, D, device="cuda", generator=g).bfloat16().requires_grad_()
    w = torch.randn(V, D, device="cuda", generator=g).bfloat16().requires_grad_()
    tokens = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32, generator=g)
    tokens[:3] = torch.tensor([V - 1, 524287, 524288])
    lp, _ = cd.head_logprobs(h, w, tokens)
    g0 = torch.rand(T, device="cuda", generator=g)
    gh, gw = torch.autograd.grad([lp], [h, w], [g0])
    hf, wf = h.detach().float(), w.detach().float()
    logp = torch.log_softmax(hf @ wf.t(), 1)
    at, used = tokens.clamp_min(0).long()[:, None], tokens >= 0
    assert (lp - torch.where(used, logp.gather(1, at)[:, 0], 0)).abs().max() < 1e-4
    d = -logp.exp_() * (g0 * used)[:, None]
    d.scatter_add_(1, at, (g0 * used)[:, None])
    # The result rounded to 2^-8; d in two parts, and float32 logits of about 20 in both.
    for got, ref, size in ((gh, d @ wf, d.abs() @ wf.abs()), (gw, d.t() @ hf, d.abs().t() @ hf.abs())):
        assert ((got.float() - ref).abs() <= 1.01 * 2.0 ** -8 * ref.abs() + 1e-4 * size + 1e-7).all()


def test_large_steps_give_the_same_bits():
    # Large tiles in all products, sums over ranges of the vocabulary and over parts.
    for T, D, V, dtype in ((8192, 512, 65536, "bf16"), (3001, 1000, 10007, "f16")):
        g = torch.Generator(device="cuda").manual_seed(25)
        h = torch.randn(T, D, device="cuda", generator=g).to(DTYPES[dtype]).requires_grad_()
        w = (torch.randn(V, D, device="cuda", generator=g) / 16).to(DTYPES[dtype]).requires_grad_()
        tokens = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32, generator=g)

        def step():
            out = cd.head_logprobs(h, w, tokens)
            return out + torch.autograd.grad(out[0].sum() + out[1].sum(), [h, w])

        first = step()
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(step(), first))
