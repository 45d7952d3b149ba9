"""Scores of token ids (tt_logprobs, tt_logprobs_grad) against their definition in 64 bits, and their refusals.

Tolerances, with e = 2^-24 (half a step of 32 bits), d_j = scale (x_j - max), E the mean under the row's probabilities:
each exp d_j is off by at most 2^-22 (the hardware's exponential) + 3 e |d_j| (three roundings on the way to its exponent) relative to itself, a
sum that one of at least 128 threads takes over its share of the row and that is then joined by at most 32 more additions adds e (n / 128 + 32):
  S = 2^-22 + e (3 E|d| + n / 128 + 32)                            relative error of sum exp d, so the absolute one of its logarithm
  logprob: S + e (3 |d_t| + 2 ln s)      lse: S + 3 e |scale max| + 2 e (ln s + |lse|)
  entropy: S + 2 e ln s + E|d| (S + 2^-22 + e (n / 128 + 36)) + 3 e E d^2 + 2 e entropy
"""
import ctypes

import numpy as np
import pytest

EPS = 2.0 ** -24
KINDS = ["bf16", "fp16", "fp32"]


@pytest.fixture(scope="module")
def tt():
    from paper_2607_29678_b200 import build
    build.build()
    import paper_2607_29678_b200 as m
    return m


def _kind(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


# ---- the definition in 64 bits ------------------------------------------------------------------------------------


def targets(ids, ids_off, n_vocab):
    """Per row: the id asked for, -1 for none, -2 for a row that is not in use."""
    ids = np.asarray(ids, dtype=np.int64)
    if ids_off is None:
        return np.where((ids >= 0) & (ids < n_vocab), ids, -1)
    t = np.full(ids.size, -2, dtype=np.int64)
    for a, b in zip(ids_off[:-1], ids_off[1:]):
        for i in range(a, b):
            nxt = ids[i + 1] if i + 1 < b else -1
            t[i] = nxt if 0 <= nxt < n_vocab else -1
    return t


def order(x):
    """The entries of a row, the larger first, equal ones by index."""
    return np.lexsort((np.arange(x.size), -(x + 0.0)))


def row_scores(x, scale, t, k):
    """dict of one row's outputs and their tolerances; x in 64 bits."""
    n = x.size
    if np.isnan(x).any() or (x == np.inf).any():
        return dict(logprob=0.0 if t < 0 else np.nan, lse=np.nan, entropy=np.nan, rank=0, top_ids=np.full(k, -1), top_logprobs=np.full(k, np.nan), tol={})
    at = order(x)
    place = np.empty(n, dtype=np.int64)
    place[at] = np.arange(n)
    rank = 0 if t < 0 else int(place[t]) + 1
    m = x.max()
    if m == -np.inf:
        return dict(logprob=0.0 if t < 0 else -np.inf, lse=-np.inf, entropy=0.0, rank=rank, top_ids=at[:k], top_logprobs=np.full(k, -np.inf), tol={})
    d = scale * (x - m)
    p = np.exp(d)
    s = p.sum()
    p /= s
    ls = np.log(s)
    low = p > 0
    e_d, e_dd = -(p[low] * d[low]).sum(), (p[low] * d[low] ** 2).sum()
    ent = ls + e_d
    S = 2.0 ** -22 + EPS * (3 * e_d + n / 128 + 32)
    lse = scale * m + ls
    lp_tol = lambda v: S + EPS * (3 * np.abs(v) + 2 * ls)  # noqa: E731
    finite = lambda v: np.where(np.isfinite(v), v, 0.0)  # noqa: E731
    return dict(logprob=0.0 if t < 0 else d[t] - ls, lse=lse, entropy=ent, rank=rank, top_ids=at[:k], top_logprobs=d[at[:k]] - ls,
                tol=dict(logprob=lp_tol(finite(d[t])) if t >= 0 else 0.0, lse=S + 3 * EPS * abs(scale * m) + 2 * EPS * (ls + abs(lse)),
                         entropy=S + 2 * EPS * ls + e_d * (S + 2.0 ** -22 + EPS * (n / 128 + 36)) + 3 * EPS * e_dd + 2 * EPS * ent, top_logprobs=lp_tol(finite(d[at[:k]]))))


def near(got, want, tol):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    plain = np.isfinite(want)
    # a log probability below what 32 bits hold (masks of the type's lowest value) may come back as -inf
    far = plain & (want < -3.0e38)
    same = np.where(far, got < -3.0e38, np.where(plain, np.abs(got - np.where(plain, want, 0.0)) <= tol, (got == want) | (np.isnan(got) & np.isnan(want))))
    return bool(np.all(same))


def check_scores(logits, ids, bufs, ids_off=None, scale=1.0, untouched=None):
    """Every row of bufs against the definition; rows not in use hold what `untouched` holds."""
    x = logits.double().cpu().numpy()
    t = targets(ids.cpu().numpy(), None if ids_off is None else ids_off.cpu().numpy(), x.shape[1])
    got = {k: v.cpu().numpy() for k, v in bufs.items()}
    k = got["top_ids"].shape[1] if "top_ids" in got else 0
    scale = float(np.float32(scale))
    for i in range(x.shape[0]):
        if t[i] == -2:
            for name in got:
                if name != "status":
                    assert np.array_equal(got[name][i], untouched[name][i], equal_nan=True), (i, name)
            continue
        w = row_scores(x[i], scale, t[i], k)
        for name in ("logprob", "lse", "entropy", "top_logprobs"):
            if name in got:
                assert near(got[name][i], w[name], w["tol"].get(name, 0.0)), (i, name, got[name][i], w[name], w["tol"].get(name))
        if "rank" in got:
            assert got["rank"][i] == w["rank"], (i, got["rank"][i], w["rank"])
        if k:
            assert np.array_equal(got["top_ids"][i], w["top_ids"]), (i, got["top_ids"][i], w["top_ids"])


def row_grad(x, scale, t, lse, ent, g, h):
    """(gradient, tolerance before the rounding to the output's type) of one row from its definition; lse and ent as handed to the kernel."""
    g = g if t >= 0 else 0.0
    if (g == 0 and h == 0) or lse < -2.0 ** 60:
        return np.zeros_like(x), np.zeros_like(x)
    lp = np.minimum(scale * x - lse, 0.0)                                 # (what the rounding of lse leaves above 0)
    p = np.exp(lp)
    lpz = np.where(p > 0, lp, 0.0)
    hot = np.zeros_like(x)
    if t >= 0:
        hot[t] = 1.0
    dx = scale * (g * (hot - p) - h * p * (lpz + ent))
    rel = 2.0 ** -22 + 4 * EPS * np.abs(lpz) + 4 * EPS                   # of p: the exponent's roundings and the hardware's exponential
    tol = scale * ((abs(g) + abs(h) * np.abs(lpz + ent)) * p * (rel + 6 * EPS) + 4 * EPS * abs(g) * hot + 3 * EPS * abs(h) * p * (np.abs(lpz) + abs(ent)))
    # a probability below the normal numbers of 32 bits (2^-126) may be 0: an error of at most itself times its factor, whose logarithm is above -104
    flushed = scale * 2.0 ** -126 * (abs(g) + abs(h) * (104 + abs(ent)))
    return dx, tol + flushed


def check_grad(logits, ids, bufs, g, h, grad, ids_off=None, scale=1.0, untouched=None):
    import torch
    x = logits.double().cpu().numpy()
    t = targets(ids.cpu().numpy(), None if ids_off is None else ids_off.cpu().numpy(), x.shape[1])
    lse, ent = bufs["lse"].double().cpu().numpy(), bufs["entropy"].double().cpu().numpy()
    got = grad.double().cpu().numpy()
    half = torch.finfo(grad.dtype).eps / 2
    least = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 0.0}[grad.dtype]     # half the smallest subnormal
    scale = float(np.float32(scale))
    for i in range(x.shape[0]):
        if t[i] == -2:
            assert np.array_equal(got[i], untouched[i]), i
            continue
        hi = 0.0 if h is None else float(h[i])
        want, tol = row_grad(x[i], scale, t[i], lse[i], ent[i], float(g[i]), hi)
        if np.isnan(lse[i]) and not (hi == 0 and (float(g[i]) == 0 or t[i] < 0)):
            assert np.isnan(got[i]).all(), i
            continue
        off = np.abs(got[i] - want) - (tol + half * (np.abs(want) + tol) + least)
        assert off.max() <= 0, (i, int(off.argmax()), got[i][off.argmax()], want[off.argmax()], tol[off.argmax()])


# ---- on the CPU: the definition itself, refusals -------------------------------------------------------------------


def test_definition_on_hand_examples():
    w = row_scores(np.log(np.array([1.0, 2.0, 4.0, 1.0])), 1.0, 3, 4)
    assert np.isclose(w["logprob"], np.log(1 / 8)) and np.isclose(w["lse"], np.log(8)) and w["rank"] == 4
    assert np.isclose(w["entropy"], -(2 / 8 * np.log(1 / 8) + 2 / 8 * np.log(2 / 8) + 4 / 8 * np.log(4 / 8)))
    assert list(w["top_ids"]) == [2, 1, 0, 3]
    assert list(targets([5, 6, 7, 8, 9], [0, 2, 2, 4], 8)) == [6, -1, -1, -1, -2]
    assert list(targets([5, -1, 9], None, 8)) == [5, -1, -1]


def test_definition_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, step = rng.normal(0, 2, 9), 1e-5
    for scale, g, h, t in ((1.0, 1.0, 0.0, 4), (0.7, -0.5, 0.3, 0), (1.3, 0.0, 1.0, -1)):
        loss = lambda y: (lambda w: (g * w["logprob"] if t >= 0 else 0.0) + h * w["entropy"])(row_scores(y, scale, t, 0))  # noqa: E731
        w = row_scores(x, scale, t, 0)
        dx, _ = row_grad(x, scale, t, w["lse"], w["entropy"], g, h)
        num = np.array([(loss(x + step * np.eye(9)[j]) - loss(x - step * np.eye(9)[j])) / (2 * step) for j in range(9)])
        assert np.abs(num - dx).max() < 1e-8


def test_refusals_without_a_device(tt):
    """Arguments are looked at before any CUDA call: the addresses here are never used."""
    L, a = tt.lib(), 0x1000

    def fwd(logits=a, dtype=0, rows=2, n=8, stride=8, scale=1.0, ids=a, off=None, docs=0, k=0, lp=a, top_i=None, top_l=None, status=a):
        return L.tt_logprobs(logits, dtype, rows, n, stride, scale, ids, off, docs, k, None, lp, None, None, None, top_i, top_l, status)

    bad = [dict(logits=None), dict(logits=a + 1), dict(logits=a + 2, dtype=2), dict(dtype=3), dict(dtype=-1), dict(n=0), dict(n=1 << 31, stride=1 << 31), dict(rows=1 << 24),
           dict(stride=7), dict(stride=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=2.0 ** 101), dict(scale=float("nan")), dict(ids=None), dict(docs=1),
           dict(lp=None), dict(status=None), dict(k=9, top_i=a, top_l=a), dict(k=33, n=64, stride=64, top_i=a, top_l=a), dict(k=1), dict(k=1, top_i=a), dict(top_i=a, top_l=a),
           dict(off=a, docs=1 << 31), dict(off=a + 4, docs=1), dict(ids=a + 2), dict(status=a + 1), dict(lp=a + 2), dict(k=1, top_i=a + 1, top_l=a), dict(k=1, top_i=a, top_l=a + 2)]
    for kw in bad:
        assert fwd(**kw) == tt.TT_ERR_ARG, kw

    def bwd(logits=a, rows=2, n=8, stride=8, lse=a, ent=None, g=a, h=None, grad=2 * a, gstride=8, status=a, dtype=0):
        return L.tt_logprobs_grad(logits, dtype, rows, n, stride, 1.0, a, None, 0, lse, ent, g, h, None, grad, gstride, status)

    for kw in [dict(lse=None), dict(g=None), dict(h=a), dict(ent=a), dict(grad=None), dict(gstride=7), dict(grad=a, gstride=9), dict(grad=2 * a + 1), dict(lse=a + 2), dict(g=a + 1), dict(h=a + 2, ent=a), dict(h=a, ent=a + 1), dict(status=None), dict(dtype=5)]:
        assert bwd(**kw) == tt.TT_ERR_ARG, kw


def test_binding_refuses_what_does_not_fit(tt):
    import torch
    x = torch.zeros((2, 8))
    bufs = tt.alloc_logprobs(2, device="cpu")
    with pytest.raises(ValueError):
        tt.logprobs(x, torch.zeros(2, dtype=torch.int32), bufs)             # not on a device
    with pytest.raises(ValueError):
        tt.logprobs(x.double(), torch.zeros(2, dtype=torch.int32), bufs)


# ---- on the GPU ----------------------------------------------------------------------------------------------------


def make_logits(kind, rows, n, seed, pad=0, shift=0, spread=2.5):
    """Random logits as a view whose rows lie n + pad entries apart, `shift` entries behind an aligned address."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    step = n + pad
    whole = torch.full((rows * step + shift,), 77.0, dtype=_kind(kind), device="cuda")
    x = whole[shift:].view(rows, step)[:, :n]
    x.copy_(torch.randn((rows, n), generator=g, device="cuda") * spread)
    return x


def make_ids(rows, n, seed, none_every=0):
    import torch
    g = torch.Generator().manual_seed(seed + 1)
    ids = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32)
    if none_every:
        ids[::none_every] = -1
    return ids.cuda()


def run_scores(tt, x, ids, k=0, ids_off=None, scale=1.0, fill=None, status=0):
    import torch
    bufs = tt.alloc_logprobs(x.shape[0], k)
    for name, v in bufs.items():
        v.fill_(-7)
    before = {name: v.cpu().numpy().copy() for name, v in bufs.items()}
    tt.logprobs(x, ids, bufs, ids_off=ids_off, scale=scale)
    torch.cuda.synchronize()
    assert int(bufs["status"].item()) == status
    return bufs, before


SHAPES = [(1, 1, 0), (1, 1, 1), (3, 2, 2), (2, 7, 5), (5, 31, 31), (4, 33, 32), (3, 255, 4), (2, 1_000, 32), (2, 4_352, 5), (7, 4_353, 20), (2, 32_257, 32), (1, 100_256, 5),
          (150, 5_003, 3), (300, 2_048, 1), (2, 200_001, 20)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_scores_match_the_definition(tt, kind, rows, n, k):
    for pad, shift, scale in ((0, 0, 1.0), (3, 1, 0.7)):
        x = make_logits(kind, rows, n, seed=rows * n + k + pad, pad=pad, shift=shift)
        ids = make_ids(rows, n, n + pad, none_every=4 if rows > 3 else 0)
        bufs, _ = run_scores(tt, x, ids, k, scale=scale)
        check_scores(x, ids, bufs, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 5, 129, 3_001, 20_000, 65_537])
def test_scores_of_masked_and_broken_rows(tt, kind, n):
    """Masks of -inf and of the type's lowest value, rows with nothing left, rows of one value, signed zeros, NaN and +inf."""
    import torch
    low, inf = torch.finfo(_kind(kind)).min, float("inf")
    x = make_logits(kind, 16, n, seed=n)
    gone = torch.rand((16, n), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") < 0.9
    x[0].masked_fill_(gone[0], -inf)
    x[1].masked_fill_(gone[1], low)
    x[2] = -inf
    x[3] = low
    x[4] = low; x[4].masked_fill_(gone[4], -inf)                           # the lowest value is all there is, beside -inf
    x[5] = 0.0; x[5, ::2] = -0.0
    x[6] = 3.0
    x[7, n // 2] = float("nan")
    x[8, n // 3] = inf
    x[9] = float("nan")
    x[10] = -inf; x[10, n - 1] = -4.0                                      # one entry left
    x[11] = -inf; x[11, n // 2] = float("nan")
    x[12] = torch.finfo(_kind(kind)).max
    x[13] = low; x[13, n // 2] = torch.finfo(_kind(kind)).max              # a distance of twice the largest value
    x[14] = inf
    x[15] = inf; x[15, 0] = -inf
    ids = make_ids(16, n, n)
    ids[10] = n - 1
    for scale in (1.0, 1.5):
        bufs, _ = run_scores(tt, x, ids, min(n, 32), scale=scale)
        if scale != 1.0 and kind != "fp16":                                # scale * max passes 32 bits: the lse is an infinity
            assert bufs["lse"][12].item() == inf and bufs["lse"][3].item() == -inf
            del bufs["lse"]
        check_scores(x, ids, bufs, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", [(6, 20_001), (160, 9_000), (900, 4_100)])
def test_masks_through_long_rows(tt, kind, rows, n):
    """Masked entries in every batch of a thread, of either kind and mixed, with the row's id masked, low or the only one left."""
    import torch
    low, inf = torch.finfo(_kind(kind)).min, float("inf")
    x = make_logits(kind, rows, n, seed=rows)
    g = torch.Generator(device="cuda").manual_seed(n)
    gone = torch.rand((rows, n), generator=g, device="cuda")
    x.masked_fill_(gone < 0.4, -inf)
    x[::2].masked_fill_(gone[::2] > 0.7, low)
    x[1::6, n // 2:] = low
    x[4::12] -= 30_000.0
    x[5::12] = torch.where(gone[5::12] < 0.5, torch.tensor(low, dtype=x.dtype, device="cuda"), torch.tensor(low, dtype=x.dtype, device="cuda") * 0.99)
    x[3::18] = -inf; x[3::18, n - 7] = 2.0
    x[7::20] = low; x[7::20, ::3] = -inf
    ids = make_ids(rows, n, rows)
    bufs, _ = run_scores(tt, x, ids, 5, scale=1.25 if kind == "fp16" else 1.0)
    check_scores(x, ids, bufs, scale=1.25 if kind == "fp16" else 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [257, 8_200, 50_001, 150_000])
def test_alternatives_where_the_largest_lie_together(tt, kind, n):
    """Sorted rows, plateaus of equal values, large values at regular distances: whatever the shares that threads take of a row."""
    import torch
    rows = []
    j = torch.arange(n, device="cuda")
    rows.append(-j.float() / n)
    rows.append(j.float() / n)
    rows.append((j // 40).float() / 64)
    rows.append((n - 1 - j).float() // 100)
    for step in (2, 8, 64, 512, 1_024, 2_048, 4_096, 8_192, 16_384):
        rows.append(torch.where(j % step == step // 2, 5.0 + (j % 1_000).float() / 128, torch.zeros((), device="cuda")))
        rows.append(torch.where((j % (8 * step)) // 8 == 1, 5.0 + (j // 8 % 61).float() / 64, torch.zeros((), device="cuda")))
    x = torch.stack(rows).to(_kind(kind))
    ids = make_ids(len(rows), n, n)
    for k in (1, 7, 32):
        bufs, _ = run_scores(tt, x, ids, k)
        check_scores(x, ids, bufs)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,off", [(12, [0, 5, 12]), (12, [0, 0, 1, 1, 9, 9]), (7, [0, 0]), (9, [0, 1, 2, 3, 4]), (5, [0]), (200, list(range(0, 191, 3)) + [190]), (70, [0] * 40 + [70])])
def test_packed_documents(tt, kind, rows, off):
    """Row i scores token i + 1 of its own document; the rows behind the last one keep what they held, gradients too."""
    import torch
    n = 515
    x = make_logits(kind, rows, n, seed=rows)
    ids = make_ids(rows, n, rows)
    toff = torch.tensor(off, dtype=torch.int64, device="cuda")
    bufs, before = run_scores(tt, x, ids, 3, ids_off=toff)
    check_scores(x, ids, bufs, ids_off=toff, untouched=before)
    g = torch.randn(rows, device="cuda")
    g[::5] = 0.0
    h = torch.randn(rows, device="cuda")
    h[::2] = 0.0
    for hh in (None, h):
        grad = torch.full_like(x, 9.0)
        tt.logprobs_grad(x, ids, bufs, g, grad, ids_off=toff, grad_entropy=hh)
        torch.cuda.synchronize()
        assert int(bufs["status"].item()) == 0
        check_grad(x, ids, bufs, g, hh, grad, ids_off=toff, untouched=np.full((rows, n), 9.0))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,n", [(1, 1), (2, 2), (3, 7), (2, 129), (5, 4_352), (7, 4_353), (2, 32_257), (40, 1_000), (1, 200_001)])
@pytest.mark.parametrize("kind", KINDS)
def test_gradient_matches_the_definition(tt, kind, rows, n):
    import torch
    for pad, shift, gpad, scale in ((0, 0, 0, 1.0), (3, 1, 5, 0.7), (5, 1, 5, 1.5)):
        x = make_logits(kind, rows, n, seed=rows * n + pad, pad=pad, shift=shift)
        ids = make_ids(rows, n, n + pad, none_every=4 if rows > 3 else 0)
        bufs, _ = run_scores(tt, x, ids, scale=scale)
        g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
        for hh in (None, h):
            whole = torch.full((rows, n + gpad), 5.0, dtype=x.dtype, device="cuda")
            grad = whole[:, :n]
            tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=hh, scale=scale)
            torch.cuda.synchronize()
            assert int(bufs["status"].item()) == 0
            check_grad(x, ids, bufs, g, hh, grad, scale=scale)
            assert bool((whole[:, n:] == 5.0).all())
        same = x.clone() if pad == 0 else x
        want = grad.clone()
        tt.logprobs_grad(same, ids, bufs, g, same, grad_entropy=h, scale=scale)          # in place of the logits
        assert torch.equal(same, want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_gradient_of_masked_and_broken_rows(tt, kind):
    import torch
    n, inf, low = 1_003, float("inf"), torch.finfo(_kind(kind)).min
    x = make_logits(kind, 8, n, seed=3)
    gone = torch.rand((8, n), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") < 0.9
    x[0].masked_fill_(gone[0], -inf)
    x[1].masked_fill_(gone[1], low)
    x[2] = -inf
    x[3] = low                                                             # fp16: a uniform row; bf16 and fp32: nothing but masks, zeros
    x[4, 17] = float("nan")
    x[5, 17] = inf
    x[6, 17] = float("nan")
    x[7] = -inf; x[7, 5] = 1.0
    ids = make_ids(8, n, 1)
    bufs, _ = run_scores(tt, x, ids)
    g, h = torch.randn(8, device="cuda"), torch.randn(8, device="cuda")
    g[6] = h[6] = 0.0                                                      # nothing is asked of the broken row: zeros
    grad = torch.full_like(x, 5.0)
    tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=h)
    check_grad(x, ids, bufs, g, h, grad)
    assert kind == "fp16" or bool((grad[3] == 0).all())
    assert bool((grad[2] == 0).all()) and bool((grad[6] == 0).all()) and bool(torch.isnan(grad[4:6].float()).all())
    assert bool((grad[0][gone[0]] == 0).sum() >= gone[0].sum() - 1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_gradient_of_rows_far_from_0_stays_finite(tt, kind):
    """Logits of a size at which lse is off by more than 1 from its rounding, and rows that the type's lowest value masks wholly, at several scales."""
    import torch
    low = torch.finfo(_kind(kind)).min
    x = make_logits(kind, 6, 700, seed=8)
    x[0] = low; x[0, ::3] = -float("inf")
    x[1] = low
    x[2] += 60_000.0 if kind == "fp16" else 3e8
    x[3] -= 60_000.0 if kind == "fp16" else 3e8
    x[4] = low; x[4, 5] = 0.25
    ids = make_ids(6, 700, 1)
    g, h = torch.ones(6, device="cuda"), torch.ones(6, device="cuda")
    for scale in (1.0, 0.01, 1.5, 1e-6):
        bufs, _ = run_scores(tt, x, ids, scale=scale)
        for hh in (None, h):
            grad = torch.full_like(x, 9.0)
            tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=hh, scale=scale)
            assert bool(torch.isfinite(grad).all()), scale
            assert float(grad[4].float().abs().sum()) <= 2.0 * scale + 1e-3 or scale == 1e-6
            check_grad(x[4:], ids[4:], {k: v[4:] for k, v in bufs.items() if k != "status"}, g[4:], None if hh is None else hh[4:], grad[4:], scale=scale)


@pytest.mark.gpu
def test_gradient_against_differences_of_the_definition(tt):
    """Central differences of the scores in 64 bits, step 1e-5: off by some 1e-9 themselves."""
    import torch
    x = make_logits("fp32", 3, 40, seed=9)
    ids = make_ids(3, 40, 2)
    bufs, _ = run_scores(tt, x, ids, scale=1.25)
    g, h = torch.tensor([1.0, -0.5, 0.25], device="cuda"), torch.tensor([0.5, 1.0, -2.0], device="cuda")
    grad = torch.zeros_like(x)
    tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=h, scale=1.25)
    xs, step = x.double().cpu().numpy(), 1e-5
    for i in range(3):
        t = int(ids[i])
        f = lambda y: float(g[i]) * row_scores(y, 1.25, t, 0)["logprob"] + float(h[i]) * row_scores(y, 1.25, t, 0)["entropy"]  # noqa: E731
        num = np.array([(f(xs[i] + step * np.eye(40)[j]) - f(xs[i] - step * np.eye(40)[j])) / (2 * step) for j in range(40)])
        lse, ent = float(bufs["lse"][i]), float(bufs["entropy"][i])
        _, tol = row_grad(xs[i], 1.25, t, lse, ent, float(g[i]), float(h[i]))
        # the lse and entropy handed over are off by at most their own tolerance: p by that much relative to itself
        w = row_scores(xs[i], 1.25, t, 0)["tol"]
        p = np.exp(1.25 * xs[i] - lse)
        more = 1.25 * p * (w["lse"] * (abs(float(g[i])) + abs(float(h[i])) * (np.abs(np.log(p) + ent) + 1)) + abs(float(h[i])) * w["entropy"])
        assert (np.abs(grad[i].double().cpu().numpy() - num) <= tol + more + 1e-8 + EPS * np.abs(num)).all()


@pytest.mark.gpu
def test_statuses(tt):
    import torch
    n = 100
    x = make_logits("bf16", 10, n, seed=1)
    ids = make_ids(10, n, 1)
    off = lambda *v: torch.tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
    wrong = ids.clone(); wrong[4] = n
    bufs, before = run_scores(tt, x, wrong, status=tt.TT_ERR_BAD_IDS)
    check_scores(x, wrong, bufs)                                           # that row counts as asked for nothing
    assert bufs["logprob"][4].item() == 0 and bufs["rank"][4].item() == 0
    run_scores(tt, x, wrong, ids_off=off(0, 4, 10))                        # the first token of a document is asked for by no row
    run_scores(tt, x, wrong, ids_off=off(0, 4))                            # nor is one behind the documents
    run_scores(tt, x, wrong, ids_off=off(0, 4, 4, 4, 10))
    run_scores(tt, x, wrong, ids_off=off(0, 3, 10), status=tt.TT_ERR_BAD_IDS)
    wrong[4] = -1
    run_scores(tt, x, wrong)
    run_scores(tt, x, wrong, ids_off=off(0, 10), status=tt.TT_ERR_BAD_IDS)
    run_scores(tt, x, ids, ids_off=off(0, 6, 5), status=tt.TT_ERR_ARG)
    run_scores(tt, x, ids, ids_off=off(1, 6, 8), status=tt.TT_ERR_ARG)
    run_scores(tt, x, ids, ids_off=off(0, -1), status=tt.TT_ERR_ARG)
    bufs, before = run_scores(tt, x, ids, 2, ids_off=off(0, 11), status=tt.TT_ERR_CAPACITY)
    for name in bufs:
        assert name == "status" or np.array_equal(bufs[name].cpu().numpy(), before[name])
    grad = torch.full_like(x, 5.0)
    tt.logprobs_grad(x, ids, bufs, torch.ones(10, device="cuda"), grad, ids_off=off(0, 11))
    torch.cuda.synchronize()
    assert int(bufs["status"].item()) == tt.TT_ERR_CAPACITY and bool((grad == 5.0).all())
    # no rows at all
    empty = tt.alloc_logprobs(0)
    empty["status"].fill_(-7)
    tt.logprobs(x[:0], ids[:0], empty)
    assert int(empty["status"].item()) == 0


@pytest.mark.gpu
def test_outputs_that_are_not_wanted(tt):
    import torch
    x = make_logits("fp16", 5, 777, seed=1)
    ids = make_ids(5, 777, 1)
    full, _ = run_scores(tt, x, ids, 4)
    for names in (["logprob"], ["logprob", "rank"], ["logprob", "entropy", "top_ids", "top_logprobs"], ["logprob", "lse"]):
        bufs = {k: torch.zeros_like(full[k]) for k in names + ["status"]}
        tt.logprobs(x, ids, bufs)
        for k in names:
            assert torch.equal(bufs[k], full[k]), k


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets(tt):
    """The last rows lie more than 2^32 bytes (and 2^31 entries) behind the first."""
    import torch
    rows, step, n = 1_030, 1 << 21, 301
    whole = torch.empty((rows, step), dtype=torch.bfloat16, device="cuda")
    x = whole[:, :n]
    x.copy_(torch.randn((rows, n), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"))
    ids = make_ids(rows, n, 1)
    bufs, _ = run_scores(tt, x, ids, 2)
    check_scores(x[-8:], ids[-8:], {k: v[-8:] if k != "status" else v for k, v in bufs.items()})
    g = torch.randn(rows, device="cuda")
    want = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    tt.logprobs_grad(x, ids, bufs, g, want)
    check_grad(x[-8:], ids[-8:], {k: v[-8:] for k, v in bufs.items() if k != "status"}, g[-8:], None, want[-8:])
    tt.logprobs_grad(x, ids, bufs, g, x)
    assert torch.equal(x, want)


@pytest.mark.gpu
def test_streams_capture_and_repetition(tt):
    """On another stream, captured and replayed on new contents, two graphs side by side; the same inputs give the same bits."""
    import torch
    x, y = make_logits("bf16", 33, 32_257, seed=1), make_logits("bf16", 33, 32_257, seed=2)
    ids = make_ids(33, 32_257, 1)
    want, _ = run_scores(tt, x, ids, 20)
    g = torch.randn(33, device="cuda")
    dx = torch.zeros_like(x)
    tt.logprobs_grad(x, ids, want, g, dx)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    live = x.clone()
    graphs = []
    for _ in range(2):
        bufs = tt.alloc_logprobs(33, 20)
        grad = torch.zeros_like(x)
        with torch.cuda.stream(side):
            tt.logprobs(live, ids, bufs, stream=side)
            tt.logprobs_grad(live, ids, bufs, g, grad)
        side.synchronize()
        assert torch.equal(grad, dx)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            tt.logprobs(live, ids, bufs)
            tt.logprobs_grad(live, ids, bufs, g, grad)
        graphs.append((graph, bufs, grad))
    live.copy_(y)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for (graph, _, _), st in zip(graphs, (side, other)):
        with torch.cuda.stream(st):
            graph.replay()
    torch.cuda.synchronize()
    ref, _ = run_scores(tt, y, ids, 20)
    for _, bufs, grad in graphs:
        for k in ref:
            assert torch.equal(bufs[k], ref[k]), k
        again = torch.zeros_like(grad)
        tt.logprobs_grad(y, ids, ref, g, again)
        assert torch.equal(grad, again)
    live.copy_(x)
    graphs[0][0].replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(graphs[0][1][k], want[k]), k


@pytest.mark.gpu
def test_binding_refuses_on_a_device(tt):
    import torch
    x = make_logits("bf16", 4, 50, seed=1)
    ids = make_ids(4, 50, 1)
    bufs = tt.alloc_logprobs(4, 2)
    for bad in (lambda: tt.logprobs(x, ids.long(), bufs), lambda: tt.logprobs(x, ids[:3], bufs), lambda: tt.logprobs(x.t(), ids, bufs), lambda: tt.logprobs(x[0], ids, bufs),
                lambda: tt.logprobs(x, ids, {**bufs, "top_ids": bufs["top_ids"][:, :1]}), lambda: tt.logprobs(x, ids, {k: v for k, v in bufs.items() if k != "top_logprobs"}),
                lambda: tt.logprobs(x, ids, {**bufs, "lse": bufs["lse"].double()}), lambda: tt.logprobs(x, ids, bufs, ids_off=torch.zeros(2, dtype=torch.int32, device="cuda")),
                lambda: tt.logprobs_grad(x, ids, bufs, bufs["lse"], x.float()), lambda: tt.logprobs_grad(x, ids, bufs, bufs["lse"][:2], x)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tt.TokTierError):
        tt.logprobs(x[:1].expand(4, 50), ids, bufs)                        # rows that lie over one another
    with pytest.raises(tt.TokTierError):
        tt.logprobs(x, ids, bufs, scale=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,rows,n,k", [("bf16", 200, 50_001, 7), ("fp32", 200, 50_001, 3), ("fp16", 1_000, 10_001, 2), ("bf16", 1_300, 9_003, 0), ("fp32", 460, 4_096, 32), ("bf16", 500, 700, 1), ("fp16", 1_500, 3_001, 4),
                                            ("bf16", 460, 65_601, 20)])
def test_every_way_a_row_is_shared_out(tt, kind, rows, n, k):
    """Rows by the hundred and thousand: CTAs of 64, 128 and 256 threads, alone and in clusters."""
    x = make_logits(kind, rows, n, seed=n)
    ids = make_ids(rows, n, n, none_every=7)
    bufs, _ = run_scores(tt, x, ids, k)
    check_scores(x, ids, bufs)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_subnormal_logits_keep_their_order(tt, kind):
    import torch
    n = 2_100
    least = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -24, "fp32": 2.0 ** -149}[kind]
    g = torch.Generator().manual_seed(3)
    x = (torch.randint(-120, 121, (4, n), generator=g).double() * least).to(_kind(kind)).cuda()
    x[3] = 0.0; x[3, 5] = -least; x[3, 7] = least; x[3, 9] = -0.0
    ids = make_ids(4, n, 3)
    ids[3] = 9
    bufs, _ = run_scores(tt, x, ids, 32)
    check_scores(x, ids, bufs)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [3, 700, 33_000])
def test_sure_rows_stay_within_their_range(tt, kind, n):
    """One entry with all of the probability: no logprob above 0, no entropy below."""
    import torch
    x = torch.full((64, n), -float("inf"), dtype=_kind(kind), device="cuda")
    ids = make_ids(64, n, 1)
    at = torch.arange(64, device="cuda")
    x[at, ids.long()] = (torch.randn(64, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda") * 25).to(_kind(kind))
    x[32:] = torch.where(torch.isinf(x[32:]), x[32:].amax(1, keepdim=True) - 30, x[32:])
    for scale in (1.0, 0.37, 4.0):
        bufs, _ = run_scores(tt, x, ids, 2, scale=scale)
        check_scores(x, ids, bufs, scale=scale)
        assert float(bufs["logprob"].max()) <= 0.0 and float(bufs["top_logprobs"].max()) <= 0.0 and float(bufs["entropy"].min()) >= 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** 100, 1e6, 300.0, 1e-3, 1e-30, 1e-42])
@pytest.mark.parametrize("kind", KINDS)
def test_extreme_scales(tt, kind, scale):
    x = make_logits(kind, 5, 4_001, seed=2)
    x[1, ::3] = -float("inf")
    ids = make_ids(5, 4_001, 4)
    bufs, _ = run_scores(tt, x, ids, 5, scale=scale)
    if scale > 1e5:                                                        # lse and log probabilities of that size: their leading digits
        del bufs["lse"]
    check_scores(x, ids, bufs, scale=scale)


@pytest.mark.gpu
def test_thousands_of_documents(tt):
    """Three steps of the search for a row's document; documents without a token between the others."""
    import torch
    rng = np.random.default_rng(5)
    lengths = rng.integers(0, 4, 5_000)
    lengths[rng.integers(0, 5_000, 1_500)] = 0
    off = np.r_[0, np.cumsum(lengths)].astype(np.int64)
    rows, n = int(off[-1]) + 3, 64
    x, ids = make_logits("bf16", rows, n, seed=1), make_ids(rows, n, 1)
    toff = torch.from_numpy(off).cuda()
    bufs, before = run_scores(tt, x, ids, 0, ids_off=toff)
    check_scores(x, ids, bufs, ids_off=toff, untouched=before)
    starts = set(off.tolist())
    wrong = ids.clone()
    wrong[[i for i in range(rows - 3) if i in starts]] = n + 7             # asked for by no row
    run_scores(tt, x, wrong, 0, ids_off=toff)
    inner = next(i for i in range(2_000, rows - 3) if i not in starts)
    wrong[inner] = n
    run_scores(tt, x, wrong, 0, ids_off=toff, status=tt.TT_ERR_BAD_IDS)


@pytest.mark.gpu
def test_two_calls_at_once(tt):
    """Nothing is shared between calls: the same buffers read on two streams, each with outputs of its own."""
    import torch
    x, y = make_logits("fp16", 700, 9_001, seed=1), make_logits("fp16", 700, 9_001, seed=2)
    ids = make_ids(700, 9_001, 1)
    want = [run_scores(tt, v, ids, 8)[0] for v in (x, y)]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [tt.alloc_logprobs(700, 8), tt.alloc_logprobs(700, 8)]
    g = torch.randn(700, device="cuda")
    grads = [torch.zeros_like(x), torch.zeros_like(y)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, v, b, d in zip(streams, (x, y), got, grads):
            with torch.cuda.stream(st):
                tt.logprobs(v, ids, b)
                tt.logprobs_grad(v, ids, b, g, d)
    torch.cuda.synchronize()
    for w, b, v, d in zip(want, got, (x, y), grads):
        for k in w:
            assert torch.equal(w[k], b[k]), k
        alone = torch.zeros_like(d)
        tt.logprobs_grad(v, ids, w, g, alone)
        assert torch.equal(alone, d)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_rows_at_the_end_of_the_memory(tt, kind):
    """Logits whose last entry is the last one of a memory segment of its own, of sizes with entries on either side of the vectors."""
    import torch
    torch.cuda.empty_cache()
    size = torch.finfo(_kind(kind)).bits // 8
    whole = torch.zeros((32 << 20) // size, dtype=_kind(kind), device="cuda")      # (a segment is a multiple of 2 MB)
    for rows, n, k in ((12, 23, 23), (1, 7, 1), (40, 1_001, 3), (3, 32_257, 20), (160, 5_003, 2), (500, 301, 5)):
        x = whole[whole.numel() - rows * n:].view(rows, n)
        x.copy_(torch.randn((rows, n), generator=torch.Generator(device="cuda").manual_seed(n), device="cuda"))
        ids = make_ids(rows, n, n, none_every=5)
        bufs, _ = run_scores(tt, x, ids, k)
        check_scores(x, ids, bufs)
        g = torch.randn(rows, device="cuda")
        grad = torch.zeros((rows, n + 1), dtype=x.dtype, device="cuda")[:, :n]
        tt.logprobs_grad(x, ids, bufs, g, grad)
        check_grad(x, ids, bufs, g, None, grad)
        want = grad.clone()
        tt.logprobs_grad(x, ids, bufs, g, x)
        assert torch.equal(x, want)


def test_16_bit_logits_are_loaded_as_integers():
    """The loads that cuda_fp16.hpp and cuda_bf16.hpp define past L1 (assembly without volatile) may be taken out of their conditions."""
    import os
    import re
    src = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_29678_b200", "csrc", "tt_scores.cuh")
    with open(src) as f:
        text = f.read()
    assert re.search(r"score_raw\(const __half\* p\) \{ return __ushort_as_half\(__ldcg\(reinterpret_cast<const unsigned short\*>\(p\)\)\); \}", text)
    assert re.search(r"score_raw\(const __nv_bfloat16\* p\) \{ return __ushort_as_bfloat16\(__ldcg\(reinterpret_cast<const unsigned short\*>\(p\)\)\); \}", text)
    for arg in re.findall(r"__ld[a-z]+\(([^()]*)", text):                  # of the others none takes the address of a logit: x, dx and e are such
        assert not re.match(r"\s*(x|dx|e)\b", arg), arg


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 700, 20_001, 150_000])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_logits_over_the_whole_range_of_the_type(tt, kind, n):
    """Distances between the logits of a row that pass 32 bits, at scales that make all of them count."""
    import torch
    top = torch.finfo(_kind(kind)).max
    g = torch.Generator(device="cuda").manual_seed(n)
    rows = 12
    x = (torch.randn((rows, n), generator=g, device="cuda").double() * 1.7e38).clamp(-top, top).to(_kind(kind))
    gone = torch.rand((rows, n), generator=g, device="cuda")
    x[1] = torch.where(gone[1] < 0.5, torch.tensor(top, dtype=x.dtype, device="cuda"), torch.tensor(-top, dtype=x.dtype, device="cuda"))
    x[2] = -top; x[2, n // 2:] = top
    x[3] = -top; x[3, n - 1] = top
    x[4:8].masked_fill_(gone[4:8] < 0.4, -float("inf"))
    x[4:8, 0] = top
    x[8] = torch.where(gone[8] < 0.5, torch.tensor(-float("inf"), device="cuda"), -gone[8] * 1e38).to(x.dtype); x[8, n - 1] = top
    ids = make_ids(rows, n, n)
    ids[:4] = n - 1
    ids[4:8] = 0
    for scale in (1.2e-38, 2e-38, 1e-37):
        bufs, _ = run_scores(tt, x, ids, min(n, 5), scale=scale)
        check_scores(x, ids, bufs, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,rows,n", [("fp32", 800, 33_001), ("fp16", 1_000, 57_345), ("bf16", 1_500, 33_001), ("bf16", 1_000, 100_257)])
def test_gradient_of_many_long_rows(tt, kind, rows, n):
    """A CTA takes several batches of a row: two of the first two sizes (5 and 4 CTAs a row), four of the others (2 and 4), on 148 SMs.  Every row equals,
    bit by bit, that of a call on few rows (a batch a CTA); some rows, with their ids at the ends of the CTAs' stretches, against the definition."""
    import torch
    x = make_logits(kind, rows, n, seed=rows + n, pad=7, shift=1)
    ids = make_ids(rows, n, n, none_every=9)
    g, h = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    g[7::50] = 0.0; h[7::50] = 0.0
    size = x.element_size()
    whole = torch.full((rows, n + 7), 5.0, dtype=x.dtype, device="cuda")
    odd = torch.full((rows, n + 12), 5.0, dtype=x.dtype, device="cuda")
    grad = whole[:, :n]
    vec, picked = 16 // size, [0, 7, rows - 1]
    for i, batches in enumerate((1, 2, 4, 6, 8)):                          # the first and the last entry of stretches that end after so many batches
        for k in (0, 1):
            row = 11 + 2 * i + k
            lead = (-(grad.data_ptr() + row * grad.stride(0) * size) % 16) // size
            at = lead + batches * 4 * 256 * vec - k
            if at < n:
                ids[row] = at
                picked.append(row)
    ids[30], ids[31] = 0, n - 1
    picked += [30, 31, rows // 2]
    bufs, _ = run_scores(tt, x, ids)
    some = torch.tensor(picked, device="cuda")
    part = {k: v[some] for k, v in bufs.items() if k != "status"}
    for hh in (None, h):
        tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=hh)
        check_grad(x[some], ids[some], part, g[some], None if hh is None else hh[some], grad[some])
        for lo in range(0, rows, 100):
            few = slice(lo, min(rows, lo + 100))
            want = torch.empty_like(x[few])
            tt.logprobs_grad(x[few], ids[few], {**{k: bufs[k][few] for k in ("lse", "entropy")}, "status": bufs["status"]}, g[few], want, grad_entropy=None if hh is None else hh[few])
            assert torch.equal(grad[few], want), lo
        tt.logprobs_grad(x, ids, bufs, g, odd[:, 3:n + 3], grad_entropy=hh)        # rows that do not lie as the logits' do
        assert torch.equal(odd[:, 3:n + 3], grad)
    assert bool((whole[:, n:] == 5.0).all()) and bool((odd[:, :3] == 5.0).all()) and bool((odd[:, n + 3:] == 5.0).all())
    tt.logprobs_grad(x, ids, bufs, g, x, grad_entropy=h)                    # in place of the logits
    assert torch.equal(x, grad)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n,k", [(6, 1, 0), (6, 37, 3), (8, 4_353, 0), (6, 200_001, 20), (6, 200_001, 0), (300, 32_257, 1), (700, 70_001, 0), (1_100, 66_000, 2), (2_500, 4_353, 0)])
def test_every_entry_counts_once(tt, kind, rows, n, k):
    """Rows of one value, 0, between masked entries: the sum is their number, exact in 32 bits, and lse and entropy are its logarithm, off by at most
    one unit of the last place (logf), which is less than what one entry more or less changes: 2^-20 and 1 / 200,001 at most."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    for share in (0.0, 0.5, 0.97):
        gone = torch.rand((rows, n), generator=g, device="cuda") < share
        gone[:, n // 2] = False
        x = torch.zeros((rows, n), dtype=_kind(kind), device="cuda").masked_fill_(gone, -float("inf"))
        ids = torch.full((rows,), n // 2, dtype=torch.int32, device="cuda")
        bufs, _ = run_scores(tt, x, ids, k)
        want = torch.log((~gone).sum(1).double())
        unit = torch.where(want > 0, torch.exp2(torch.floor(torch.log2(want.clamp(min=2.0 ** -60))) - 23), 0.0)
        for name in ("lse", "entropy", "logprob"):
            off = (bufs[name].double() * (-1 if name == "logprob" else 1) - want).abs()
            assert bool((off <= unit).all()), (share, name, float(off.max()))
        assert torch.equal(bufs["rank"].long(), 1 + (~gone[:, :n // 2]).sum(1))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
def test_gradient_against_the_formula_from_the_logits_alone(tt, kind):
    """Softmax, entropy and gradient in 64 bits; what the kernel is handed (lse and entropy in 32 bits) counts towards the tolerance: p is off by expm1 of what its
    logarithm is off by.  Rows that the type's lowest value masks wholly are uniform, in bf16 and fp32 with a gradient of zeros (their lse, below -2^60,
    says nothing of their number), in fp16 with that of a uniform row."""
    import torch
    n, low = 1_501, torch.finfo(_kind(kind)).min
    x = make_logits(kind, 10, n, seed=4)
    gone = torch.rand((10, n), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda") < 0.6
    x[1].masked_fill_(gone[1], -float("inf"))
    x[2].masked_fill_(gone[2], low)
    x[3] += 100.0
    x[4] -= 3_000.0
    x[5] = low
    x[6] = low; x[6].masked_fill_(gone[6], -float("inf"))
    ids = make_ids(10, n, 1)
    g, h = torch.randn(10, device="cuda"), torch.randn(10, device="cuda")
    half = torch.finfo(x.dtype).eps / 2
    least = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 0.0}[x.dtype]
    xs = x.double().cpu().numpy()
    for scale in (1.0, 0.75):
        bufs, _ = run_scores(tt, x, ids, scale=scale)
        grad = torch.full_like(x, 9.0)
        tt.logprobs_grad(x, ids, bufs, g, grad, grad_entropy=h, scale=scale)
        got = grad.double().cpu().numpy()
        for i in range(10):
            t = int(ids[i])
            z = scale * xs[i]
            count = int((xs[i] == low).sum())
            if i in (5, 6):
                assert abs(float(bufs["entropy"][i]) - np.log(count)) <= 2.0 ** -20
                if kind != "fp16":
                    assert (got[i] == 0).all()
                    continue
            m = z.max()
            lse = m + np.log(np.exp(z - m).sum())
            p, L = np.exp(z - lse), np.where(np.isfinite(z), z - lse, 0.0)
            ent = -(p[p > 0] * L[p > 0]).sum()
            w = row_scores(xs[i], scale, t, 0)["tol"]
            hot = np.zeros(n); hot[t] = 1.0
            gi, hi = float(g[i]), float(h[i])
            want = scale * (gi * (hot - p) - hi * p * (np.where(p > 0, L, 0.0) + ent))
            L = np.where(p > 0, L, 0.0)
            dL = w["lse"] + EPS * (2 * np.abs(L) + 2 * abs(lse))           # of ln p: the lse handed over, its own rounding, that of the multiply-add
            rel = np.expm1(dL + 2.0 ** -22 + 4 * EPS * np.abs(L))           # of p: and the hardware's exponential of it
            tol = scale * (abs(gi) * p * rel + abs(hi) * p * ((np.abs(L) + ent) * rel + (dL + w["entropy"] + EPS * ent) * (1 + rel)))
            tol += scale * 8 * EPS * (abs(gi) * (p + hot) + abs(hi) * p * (np.abs(L) + ent)) * (1 + rel) + scale * 2.0 ** -126 * (abs(gi) + abs(hi) * (104 + ent))
            off = np.abs(got[i] - want) - (tol + half * (np.abs(want) + tol) + least)
            assert off.max() <= 0, (i, scale, int(off.argmax()), got[i][off.argmax()], want[off.argmax()], tol[off.argmax()])


def test_streams_of_a_torch_without_the_private_call(tt, monkeypatch):
    """The current stream's address, by the private call where there is one and by the public one where there is not; a stream of the caller's."""
    import types
    import torch
    seen = []
    monkeypatch.setattr(tt, "_lib", types.SimpleNamespace(tt_f=lambda *a: seen.append(a) or tt.TT_OK))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: types.SimpleNamespace(cuda_stream=100 + index))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 200 + index, raising=False)
    tt._call("tt_f", 1, None, (7,), (8,))
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    tt._call("tt_f", 1, None, (7,), (8,))
    tt._call("tt_f", 1, types.SimpleNamespace(cuda_stream=300, device=types.SimpleNamespace(index=1)), (7,), (8,))
    assert seen == [(7, 201, 8), (7, 101, 8), (7, 300, 8)]
    with pytest.raises(ValueError):
        tt._call("tt_f", 1, types.SimpleNamespace(cuda_stream=300, device=types.SimpleNamespace(index=0)), (7,), (8,))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_a_row_of_as_many_entries_as_there_may_be(tt, kind):
    """2^31 - 1 logits, all but a thousand of them masked: their places are told apart up to the last one, gradient included (in place)."""
    import torch
    n = 2**31 - 1
    x = torch.full((1, n), -float("inf"), dtype=_kind(kind), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    at = torch.cat([torch.randint(0, n, (1_000,), generator=g, device="cuda"), torch.tensor([0, 1, 2**30 - 1, 2**30, n - 2, n - 1], device="cuda")]).unique()
    x[0, at] = torch.randn(at.numel(), generator=g, device="cuda").to(x.dtype)
    x[0, -1] = 6.0
    small = x[0, at].double().cpu().numpy()
    place = at.cpu().numpy()
    for t in (0, 500, at.numel() - 1):
        ids = torch.tensor([int(place[t])], dtype=torch.int32, device="cuda")
        bufs, _ = run_scores(tt, x, ids, 32)
        w = row_scores(small, 1.0, t, 32)
        assert int(bufs["rank"]) == w["rank"] and np.array_equal(bufs["top_ids"][0].cpu().numpy(), place[w["top_ids"]])
        for name in ("logprob", "lse", "entropy", "top_logprobs"):
            assert near(bufs[name][0].cpu().numpy(), w[name], w["tol"][name]), name
    one, h = torch.ones(1, device="cuda"), torch.full((1,), 0.5, device="cuda")
    part = {k: v for k, v in bufs.items() if k != "status"}
    tt.logprobs_grad(x, ids, bufs, one, x, grad_entropy=h)
    assert int(x.count_nonzero()) <= at.numel()
    check_grad(torch.from_numpy(small)[None], torch.tensor([t]), part, one, h, x[:, at])
