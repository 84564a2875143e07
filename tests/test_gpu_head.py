"""sample, logit_error and orthogonalize against their definitions in 64 bits, at the sizes, masks and settings where they can
go wrong, and together as they are used."""
import math

import numpy as np
import pytest

import head_reference as ref

pytestmark = pytest.mark.gpu


def _tdtype(dtype):
    import torch

    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _rows(z, dtype, pad=0, fill=math.nan):
    """numpy rows -> a device tensor of the type whose rows are `pad` columns further apart (which hold `fill`), and what it holds."""
    import torch

    n, C = z.shape
    t = torch.full((n, C + pad), fill, dtype=_tdtype(dtype), device="cuda")
    t[:, :C] = torch.from_numpy(np.ascontiguousarray(z)).cuda().to(t.dtype)
    return t[:, :C], t[:, :C].double().cpu().numpy()


def _f32(v):
    return float(np.float32(v))


# ---- sample -----------------------------------------------------------------------------------------------------

PLAIN = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


def _check_sample(z, u, dtype, pad=0, rows_as_tensors=False, **how):
    import torch
    from paper_2510_02470_amd.binding import sample

    how = dict(PLAIN, **how)
    zd, zh = _rows(z, dtype, pad)
    ud = torch.tensor(np.asarray(u, dtype=np.float32)).cuda()
    n = len(z)
    per_row = {k: np.broadcast_to(np.asarray(v, dtype=np.int32 if k == "top_k" else np.float32), (n,)) for k, v in how.items()}
    call = {}
    for k, v in how.items():
        call[k] = torch.from_numpy(per_row[k].copy()).cuda() if rows_as_tensors or np.ndim(v) else v
    labels, logp = sample(zd, ud, **call)
    labels, logp = labels.cpu().numpy(), logp.cpu().numpy()
    for i in range(n):
        T, K, P, M = (float(per_row[k][i]) for k in ("temperature", "top_k", "top_p", "min_p"))
        j, lp = ref.sample_row(zh[i], float(np.float32(u[i])), T, int(K), P, M)
        assert labels[i] == j, (i, labels[i], j)
        # one rounding to fp32 of what 64 bits give
        assert (math.isnan(lp) and math.isnan(logp[i])) or abs(logp[i] - lp) <= 2.0 ** -24 * abs(lp) + 1e-12, (i, logp[i], lp)
    return labels


def _some_rows(n, C, seed, scale=3.0):
    rng = np.random.default_rng(seed)
    z = scale * rng.standard_normal((n, C))
    z[:, rng.integers(0, C, size=min(C, 5))] += 6.0
    return z, rng.random(n, dtype=np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(1, 1), (3, 2), (9, 7), (5, 63), (5, 64), (40, 1000), (3, 8191), (3, 8193), (2, 65_537), (2, 131_073),
                                 (1, 300_007), (1, 1_048_576)])
def test_sample_every_setting(n, C, dtype):
    z, u = _some_rows(n, C, 1000 * n + C)
    for how in (dict(), dict(temperature=0.7, top_k=max(1, C // 3)), dict(top_p=0.9), dict(temperature=1.4, min_p=0.05),
                dict(temperature=0.0), dict(temperature=0.9, top_k=50, top_p=0.8, min_p=0.01)):
        _check_sample(z, u, dtype, **how)
    _check_sample(z, u, dtype, pad=3, rows_as_tensors=True, temperature=1.2, top_k=min(C, 20), top_p=0.95, min_p=0.001)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_settings_of_every_row(dtype):
    n, C = 64, 5003
    z, u = _some_rows(n, C, 5)
    i = np.arange(n)
    _check_sample(z, u, dtype, pad=1, temperature=np.array([0.0, 0.3, 1.0, 2.5])[i % 4], top_k=np.array([0, 1, 40, 6000, -2])[i % 5],
                  top_p=np.array([1.0, 0.9, 0.2])[i % 3], min_p=np.array([0.0, 0.1])[i % 2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 700, 40_000])
def test_sample_ties(C, dtype):
    """Equal logits: the lower class first, at the border of top-k, of top-p and of both."""
    rng = np.random.default_rng(C)
    z = rng.integers(-2, 2, size=(24, C)).astype(np.float64)
    z[0] = 0.0
    z[1] = np.where(np.arange(C) % 2, -0.0, 0.0)
    u = rng.random(24, dtype=np.float32)
    for how in (dict(), dict(top_k=1), dict(top_k=C // 3 + 1), dict(top_p=0.5), dict(top_p=0.3, top_k=C // 2 + 1), dict(temperature=0.0),
                dict(min_p=1.0), dict(temperature=0.25, top_p=0.99)):
        _check_sample(z, u, dtype, **how)


@pytest.mark.parametrize("how", [dict(), dict(top_k=7), dict(top_p=0.6), dict(min_p=0.2), dict(top_k=9, top_p=0.7, min_p=0.01)])
def test_sample_draws_every_kept_class_as_often_as_it_should(how):
    """One row, random numbers evenly over [0, 1): the borders between the labels are where the weights put them, and
    nothing that is not kept is drawn."""
    z, _ = _some_rows(1, 300, 17)
    u = (np.arange(4096) / 4096).astype(np.float32)
    labels = _check_sample(np.repeat(z, len(u), 0), u, "f32", temperature=1.5, **how)
    kept, w = ref.kept_classes(_rows(z, "f32")[1][0], 1.5, how.get("top_k", 0), _f32(how.get("top_p", 1.0)), _f32(how.get("min_p", 0.0)))
    assert set(labels) <= set(kept) and (np.diff(labels) >= 0).all()
    share = w[kept] / w[kept].sum()
    assert np.abs(np.array([(labels == j).mean() for j in kept]) - share).max() <= 1 / 4096


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(3, 900), (3, 5000), (3, 40_000), (300, 20_000)])
def test_sample_borders_among_many_classes(n, C, dtype):
    """Top-k of more classes than are ranked one by one, borders of top-p in flat rows (a bin holds thousands), few distinct values."""
    rng = np.random.default_rng(n + C)
    z = 0.01 * rng.standard_normal((n, C))
    z[1] = rng.integers(0, 3, C)
    z[2] = 30 * rng.standard_normal(C)
    u = rng.random(n, dtype=np.float32)
    for how in (dict(top_k=C // 2), dict(top_k=C - 1, top_p=0.9), dict(top_p=0.7), dict(top_p=0.7, min_p=0.999), dict(top_k=C // 3, top_p=0.5, min_p=0.2),
                dict(temperature=0.02, top_p=0.8)):
        _check_sample(z, u, dtype, **how)


def _rows_of_values(kind, n, C, rng):
    """Long rows whose values repeat, or are of magnitudes that only some rows have."""
    z = 2.0 * rng.standard_normal((n, C))
    some = lambda count: (np.arange(n)[:, None], np.stack([rng.permutation(C)[:count] for _ in range(n)]))
    if kind == "few values":
        z = rng.integers(-4, 5, size=(n, C)) + 0.5
    elif kind == "one value":
        z = np.repeat(np.resize([0.5, -3.0, 0.0, 130.0], n)[:, None], C, axis=1)
    elif kind == "whole numbers":
        z = np.round(z)  # zeros among them
    elif kind == "some near zero":
        z[some(300)] = 0.001 * rng.standard_normal((n, 300))
    elif kind == "near zero":
        z *= 0.0005
    elif kind == "most weight near zero":
        z = -6.0 + 0.1 * z
        z[some(700)] = 0.001 * rng.standard_normal((n, 700))
        z[some(3)] = 1.0
    elif kind == "negative":
        z = -1.0 - np.abs(z)
    elif kind == "great":
        z[some(4)] = 127.0 + 4.0 * rng.random((n, 4))
    elif kind == "far below":
        z[some(C // 2)] = np.resize([-128.0, -150.0, -3.3e38, -np.inf], n)[:, None]
    elif kind == "no distribution":
        z[np.arange(n), rng.integers(0, C, size=n)] = np.resize([np.nan, np.inf, -np.inf], n)
    return z


@pytest.mark.parametrize("kind", ["few values", "one value", "whole numbers", "some near zero", "near zero", "most weight near zero", "negative",
                                  "great", "far below", "no distribution"])
@pytest.mark.parametrize("n,C", [(8, 9001), (8, 40_000), (260, 33_001)])
def test_sample_values_of_long_rows(n, C, kind):
    rng = np.random.default_rng(C)
    z = _rows_of_values(kind, n, C, rng)
    u = rng.random(n, dtype=np.float32)
    for dtype in ("bf16", "f32") if n < 100 else ("bf16",):
        _check_sample(z, u, dtype, pad=3, rows_as_tensors=True, temperature=np.resize([1.0, 0.5, 30.0, 1.0, math.inf, 2.0, 1e-40], n),
                      top_p=np.resize([0.9, 1.0, 0.3, 0.02, 0.6], n), min_p=np.resize([0.0, 0.0, 0.0, 0.1], n), top_k=np.resize([0, C, 0], n))
    if n < 100:
        for p in (0.0, 0.05, 0.5, 0.97):
            _check_sample(z, u, "bf16", top_p=p)


def test_sample_random_numbers_at_and_beyond_the_ends():
    z, _ = _some_rows(8, 500, 3)
    z[:, 490:] = -np.inf  # the last class with a weight is not the last class
    u = np.array([0.0, -0.0, -1.0, 1.0 - 2.0 ** -24, 1.0, 7.5, np.inf, np.nan], dtype=np.float32)
    for how in (dict(), dict(top_k=3), dict(top_p=0.4)):
        _check_sample(np.repeat(z[:1], 8, 0), u, "f32", **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_masked_rows(dtype):
    """-inf, the type's lowest value, rows of nothing else, NaN and +inf; unusual temperatures."""
    import torch

    low = float(torch.finfo(_tdtype(dtype)).min)
    z, _ = _some_rows(16, 2000, 11)
    rng = np.random.default_rng(2)
    z[rng.random(z.shape) < 0.5] = -np.inf
    z[0] = -np.inf
    z[1] = low
    z[2, 1:] = low
    z[3, 1999] = np.nan
    z[4, 0] = np.inf
    z[5] = -np.inf
    z[5, 1234] = -3.0
    z[6, :] = -np.inf
    z[6, 7] = low
    z[7, 0] = -low
    u = rng.random(16, dtype=np.float32)
    for how in (dict(), dict(top_k=1500), dict(top_k=2), dict(top_p=0.9), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=math.nan),
                dict(min_p=0.5), dict(min_p=2.0), dict(min_p=math.nan), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan),
                dict(temperature=1e-30), dict(temperature=1e30), dict(temperature=math.inf)):
        labels = _check_sample(z, u, dtype, **how)
        assert list(labels[[0, 3, 4]]) == [-1, -1, -1]


def test_sample_rows_far_apart():
    """Offsets beyond 2^32 elements."""
    import torch
    from paper_2510_02470_amd.binding import logit_error, sample

    C, ld, n = 1001, (1 << 28) + 1, 18
    big = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((n, C), (ld, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    z.copy_(torch.randn(n, C, generator=g, device="cuda"))
    u = torch.rand(n, generator=g, device="cuda")
    near = z.contiguous()
    for a, b in zip(sample(z, u, top_p=0.9), sample(near, u, top_p=0.9)):
        assert torch.equal(a, b)
    y = sample(near, u)[0]
    E, loss = logit_error(near, y)
    far, loss2 = logit_error(z, y, out=z)
    assert far.data_ptr() == z.data_ptr() and torch.equal(far, E) and torch.equal(loss, loss2)


# ---- logit_error ------------------------------------------------------------------------------------------------

def _check_error(z, y, dtype, w=None, pad=0, e_dtype=None, in_place=False):
    import torch
    from paper_2510_02470_amd.binding import logit_error

    e_dtype = e_dtype or dtype
    zd, zh = _rows(z, dtype, pad)
    n, C = zh.shape
    yd = torch.tensor(y, dtype=torch.int32, device="cuda")
    wd = None if w is None else torch.tensor(w, dtype=torch.float32, device="cuda")
    wh = np.ones(n) if w is None else wd.double().cpu().numpy()
    guard = torch.full((n, C + 5), 7.0, dtype=_tdtype(e_dtype), device="cuda")
    out = zd if in_place else guard[:, :C]
    E, loss = logit_error(zd, yd, weights=wd, out=out)
    assert E.data_ptr() == out.data_ptr()
    if not in_place:
        assert bool((guard[:, C:] == 7.0).all())
    E, loss = E.double().cpu().numpy(), loss.double().cpu().numpy()
    want, want_loss, miss = ref.logit_error(zh, y, wh)
    # fp32: the difference to the maximum is rounded once (2^-24 of it), exp and the rest of a term and its factor take 8 half
    # steps, a sum of positive terms one for each addition on the longest way (C / 1024 and 24 of the trees)
    steps = 32 + C / 1024
    with np.errstate(invalid="ignore"):
        d = np.where(np.isfinite(zh), zh.max(1, initial=-1e30, where=np.isfinite(zh))[:, None] - zh, 0.0)
    rel = (d + steps + d.max(1, keepdims=True, initial=0, where=want != 0) * 0) * 2.0 ** -24
    for i in range(n):
        if np.isnan(want_loss[i]):
            assert np.isnan(loss[i]) and np.isnan(E[i]).all(), i
            continue
        # (the sum's terms have their own differences: weighted with the terms, at most ln C + 1 and what the label has)
        dy = d[i, y[i]] if 0 <= y[i] < C else 0.0
        r = rel[i] + (math.log(C) + 1 + dy) * 2.0 ** -24
        tol = np.abs(want[i]) * (r + ref.HALF_STEP[e_dtype]) + 1e-37 * (1 + abs(wh[i]))
        if np.isinf(want_loss[i]):
            assert loss[i] == np.inf
        else:
            assert abs(loss[i] - want_loss[i]) <= miss[i] * (steps + math.log(C) + 1 + 2 * dy) * 2.0 ** -24 + abs(want_loss[i]) * 2.0 ** -24 + 1e-37, i
        bad = ~(np.abs(E[i] - want[i]) <= tol)
        assert not bad.any(), (i, np.flatnonzero(bad)[:5], E[i][bad][:5], want[i][bad][:5])


@pytest.mark.parametrize("dtype,e_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n,C,pad", [(1, 1, 0), (4, 2, 1), (9, 7, 0), (5, 63, 0), (70, 64, 3), (33, 1000, 0), (7, 1001, 0), (3, 8191, 2), (2, 16_385, 0),
                                     (2, 65_537, 1), (1, 131_073, 0), (1, 1_048_576, 0)])
def test_logit_error(n, C, pad, dtype, e_dtype):
    rng = np.random.default_rng(n * 7919 + C)
    z, _ = _some_rows(n, C, n + C)
    y = rng.integers(0, C, n)
    y[::2] = z[::2].argmax(1)
    if n > 2:
        y[2] = -1
    _check_error(z, y, dtype, pad=pad, e_dtype=e_dtype)
    _check_error(z + 50.0, y, dtype, w=rng.random(n) * 3 - 1, pad=pad, e_dtype=e_dtype, in_place=dtype == e_dtype)


@pytest.mark.parametrize("n,C,dtype", [(300, 33_001, "f32"), (300, 51_200, "f32"), (260, 70_001, "bf16"), (3, 140_001, "bf16"), (40, 70_000, "f32"),
                                       (257, 131_080, "bf16")])
def test_logit_error_of_long_rows(n, C, dtype):
    """Rows that are kept in registers and LDS, or read twice, by one work-group or several."""
    import torch
    from paper_2510_02470_amd.binding import logit_error

    g = torch.Generator(device="cuda").manual_seed(C)
    z = (3 * torch.randn(n, C, generator=g, device="cuda")).to(_tdtype(dtype))
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    y[0], y[1], y[2] = 0, C - 1, -1
    w = torch.rand(n, generator=g, device="cuda") + 0.5
    E, loss = logit_error(z, y, weights=w, dtype=torch.float32)
    F, loss2 = logit_error(z, y, weights=w)
    x = z.double()
    total = torch.logsumexp(x, 1, keepdim=True)
    p = torch.exp(x - total)
    i = torch.arange(n, device="cuda")
    some = (y >= 0).double()
    want_loss = some * (total[:, 0] - x[i, y.long().clamp(min=0)])
    p[i, y.long().clamp(min=0)] -= 1.0
    p *= (w.double() * some)[:, None]
    # the terms' differences to the maximum are below 40; 32 + C / 512 additions and roundings, and the two sides of p - 1
    tol = p.abs() * (40 + 8 + 32 + C / 512) * 2.0 ** -24 + 2.0 ** -50
    assert bool(((E.double() - p).abs() <= tol).all())
    assert bool(((loss.double() - want_loss).abs() <= want_loss * 2.0 ** -24 + (80 + C / 512) * 2.0 ** -24).all())
    assert bool(((F.double() - p).abs() <= tol + p.abs() * ref.HALF_STEP[dtype]).all()) and float((loss - loss2).abs().max()) <= 2.0 ** -16
    in_place = z.clone()
    H, loss3 = logit_error(in_place, y, weights=w, out=in_place)
    assert float((H.double() - F.double()).abs().max()) <= 2 * ref.HALF_STEP[dtype] and float((loss3 - loss2).abs().max()) <= 2.0 ** -16


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logit_error_keeps_the_digits_of_learnt_examples(dtype):
    z, _ = _some_rows(8, 3000, 9)
    y = np.arange(8) * 11
    z[np.arange(8), y] = 15.0 + np.arange(8)  # the label's probability is 1 - 1e-3 .. 1 - 1e-6
    _check_error(z, y, dtype, e_dtype="f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [40, 3001])
def test_logit_error_masked_rows(C, dtype):
    import torch

    low = float(torch.finfo(_tdtype(dtype)).min)
    z, _ = _some_rows(12, C, 4)
    rng = np.random.default_rng(3)
    z[rng.random(z.shape) < 0.4] = -np.inf
    y = rng.integers(0, C, 12)
    z[np.arange(12), y] = 1.0
    z[0] = -np.inf              # nothing is possible
    z[1, y[1]] = -np.inf        # the label is not
    z[2] = -np.inf
    z[2, y[2]] = -5.0           # only the label is
    z[3] = low
    z[4, (y[4] + 1) % C] = np.nan
    z[5, y[5]] = np.inf
    y[6] = C                    # no such class
    z[7] = np.nan
    y[7] = -1                   # without a label nothing is looked at
    z[8, (y[8] + 1) % C] = -low
    y[9] = -2 ** 31
    _check_error(z, y, dtype, e_dtype="f32")
    _check_error(z, y, dtype, in_place=True)


@pytest.mark.parametrize("C", [9, 1000])
def test_logit_error_is_the_gradient_of_its_loss(C):
    """Against differences of the loss (64 bits) in random directions."""
    import torch
    from paper_2510_02470_amd.binding import logit_error

    g = torch.Generator(device="cuda").manual_seed(C)
    z = 2 * torch.randn(16, C, generator=g, device="cuda")
    y = torch.randint(0, C, (16,), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand(16, generator=g, device="cuda") + 0.5
    E, _ = logit_error(z, y, weights=w)
    v = torch.randn(16, C, generator=g, device="cuda", dtype=torch.float64)
    h = 1e-4

    def loss(x):
        return w.double() * (torch.logsumexp(x, 1) - x.gather(1, y.long()[:, None])[:, 0])

    slope = (loss(z.double() + h * v) - loss(z.double() - h * v)) / (2 * h)
    # differences are off by h^2 / 6 of the third derivative, at most |v|^3 <= 6^3; E by some fp32 steps of its terms
    assert float((slope - (E.double() * v).sum(1)).abs().max()) <= h * h * 36 * 1.5 + 6 * 1.5 * 2 * 60 * 2.0 ** -24


def test_logit_error_without_one_of_its_outputs():
    import ctypes as C

    import torch
    from paper_2510_02470_amd import binding

    z = torch.randn(5, 77, device="cuda")
    y = torch.arange(5, dtype=torch.int32, device="cuda")
    E, loss = binding.logit_error(z, y)
    L = binding.lib()
    st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    E2, loss2 = torch.zeros_like(E), torch.zeros_like(loss)
    p = lambda t: C.c_void_p(t.data_ptr())
    assert L.sage_logit_error(p(z), 0, 5, 77, 77, p(y), None, None, 0, 77, p(loss2), st) == 0
    assert L.sage_logit_error(p(z), 0, 5, 77, 77, p(y), None, p(E2), 0, 77, None, st) == 0
    assert torch.equal(E, E2) and torch.equal(loss, loss2)


def test_rows_do_not_depend_on_the_batch():
    """Few rows are shared between more work-groups than many are: the answers are the same, bit for bit."""
    import torch
    from paper_2510_02470_amd.binding import logit_error, sample

    for dtype in (torch.float32, torch.bfloat16):
        for C in (999, 33_000, 150_001):
            g = torch.Generator(device="cuda").manual_seed(C)
            z = (3 * torch.randn(300, C, generator=g, device="cuda")).to(dtype)
            u = torch.rand(300, generator=g, device="cuda")
            many = sample(z, u, top_p=0.95)
            for n in (1, 5, 40):
                few = sample(z[:n], u[:n], top_p=0.95)
                assert torch.equal(few[0], many[0][:n]) and torch.equal(few[1], many[1][:n])


# ---- orthogonalize ----------------------------------------------------------------------------------------------

MUON, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


def _gradient(m, n, seed):
    rng = np.random.default_rng(seed)
    r = max(1, min(m, n) // 2)
    G = (rng.standard_normal((m, r)) * np.arange(1, r + 1) ** -0.5) @ rng.standard_normal((r, n))
    return 1e-3 * (G + 0.2 * rng.standard_normal((m, n)))


def _check_ortho(G, dtype, steps=5, coefficients=MUON, eps=1e-7, scale=1.0, layout="rows"):
    """G: batch x rows x cols, numpy. layout: rows next to each other, "padded" rows, "columns" next to each other, "in place"."""
    import torch
    from paper_2510_02470_amd.binding import orthogonalize

    b, m, n = G.shape
    td = _tdtype(dtype)
    if layout == "padded":
        hold = torch.full((b, m + 1, n + 3), math.nan, dtype=td, device="cuda")
        Gd = hold[:, :m, :n]
    elif layout == "columns":
        Gd = torch.empty((b, n, m), dtype=td, device="cuda").transpose(1, 2)
    else:
        Gd = torch.empty((b, m, n), dtype=td, device="cuda")
    Gd.copy_(torch.from_numpy(np.ascontiguousarray(G)).cuda())
    Gh = Gd.double().cpu().numpy()
    given = Gd.clone()
    out = None
    if layout == "in place":
        out = Gd
    elif layout == "padded":
        guard = torch.full((b, m + 2, n + 1), 7.0, dtype=td, device="cuda")
        out = guard[:, :m, :n]
    res = orthogonalize(Gd, steps=steps, coefficients=coefficients, eps=eps, scale=scale, out=out)
    if layout != "in place":
        assert torch.equal(Gd, given) or not torch.isfinite(given).all()
    else:
        assert res.data_ptr() == Gd.data_ptr()
    if layout == "padded":
        assert bool((guard[:, m:] == 7.0).all()) and bool((guard[:, :, n:] == 7.0).all())
    assert res.shape == Gd.shape and res.dtype == td
    got = res.double().cpu().numpy()
    triples = coefficients if not np.isscalar(coefficients[0]) else [coefficients] * steps
    triples = [[_f32(v) for v in t] for t in triples]
    for i in range(b):
        want, norms = ref.orthogonalize(Gh[i], triples, _f32(eps), _f32(scale))
        tol = ref.orthogonalize_bound(norms, triples, scale, m * n) + 1.01 * ref.HALF_STEP[dtype] * np.linalg.norm(want)
        err = np.linalg.norm(got[i] - want)
        assert err <= tol, (i, err, tol, np.linalg.norm(want))
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 300), (300, 1), (2, 3), (7, 5), (16, 16), (33, 64), (64, 256), (100, 333), (129, 257), (300, 128), (128, 129),
                                 (500, 90), (256, 1024), (1000, 2049), (770, 770)])
def test_orthogonalize(m, n, dtype):
    _check_ortho(_gradient(m, n, m * 31 + n)[None], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["padded", "columns", "in place"])
@pytest.mark.parametrize("m,n", [(5, 9), (130, 70), (64, 200), (140, 300)])
def test_orthogonalize_layouts(m, n, layout, dtype):
    _check_ortho(np.stack([_gradient(m, n, s) for s in range(3)]), dtype, layout=layout)


@pytest.mark.parametrize("m,n", [(24, 40), (200, 150)])
def test_orthogonalize_steps_and_coefficients(m, n):
    G = _gradient(m, n, 8)[None]
    for steps in (1, 2, 3, 8):
        _check_ortho(G, "f32", steps=steps)
        _check_ortho(G, "f32", steps=steps, coefficients=CUBIC)
    _check_ortho(G, "f32", steps=4, coefficients=[MUON, MUON, (2.0, -1.5, 0.5), CUBIC])
    _check_ortho(G, "f32", steps=2, coefficients=[(0.0, 0.0, 0.0), MUON])
    _check_ortho(G, "f32", steps=1, coefficients=(20.0, 0.5, 0.25), scale=-3.5)
    _check_ortho(G, "f32", eps=0.05, scale=0.2)
    _check_ortho(G, "bf16", eps=0.0, scale=100.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(20, 30), (150, 140)])
def test_orthogonalize_unusual_matrices(m, n, dtype):
    rng = np.random.default_rng(m)
    g = _gradient(m, n, 2)
    one = np.outer(rng.standard_normal(m), rng.standard_normal(n))  # rank one
    spike = np.zeros((m, n))
    spike[m // 2, n // 3] = -4.0
    stack = np.stack([np.zeros((m, n)), g * 1e30, g * 1e-25, one, spike, np.ones((m, n)), np.eye(m, n)])
    got = _check_ortho(stack, dtype, eps=0.0)
    assert not got[0].any()
    _check_ortho(stack, dtype, eps=1e-7)


@pytest.mark.parametrize("b,m,n,dtype", [
    (1, 1800, 1930, "f32"),      # tiles of 128 x 128, the left-over ones in parts
    (1, 1930, 1800, "bf16"),
    (1, 4000, 3600, "f32"),      # tiles of 256 x 256 for one of the products
    (1, 512, 16_400, "bf16"),
    (3, 700, 1300, "f32"),
    (30, 513, 500, "bf16"),      # a batch of them
    (60, 200, 300, "f32"),
    (20, 65, 129, "f32"),        # just beyond the smallest ones
    (700, 64, 512, "bf16"),      # the largest of the smallest ones, and more of them than have helping waves
    (600, 64, 512, "f32"),
])
def test_orthogonalize_large(b, m, n, dtype):
    """Against 64-bit products on the GPU (numpy would take minutes)."""
    import torch
    from paper_2510_02470_amd.binding import orthogonalize

    g = torch.Generator(device="cuda").manual_seed(b + m + n)
    G = (torch.randn(b, m, n, generator=g, device="cuda") * torch.rand(n, generator=g, device="cuda")).to(_tdtype(dtype))
    out = orthogonalize(G, scale=0.5)
    again = orthogonalize(G, scale=0.5)
    assert torch.equal(out, again)
    for i in sorted({0, b // 2, b - 1}):
        X = G[i].double() if m <= n else G[i].double().T.contiguous()
        X = X / (torch.linalg.vector_norm(X) + _f32(1e-7))
        norms = []
        for _ in range(5):
            norms.append(float(torch.linalg.vector_norm(X)))
            A = X @ X.T.contiguous()
            X = _f32(MUON[0]) * X + (_f32(MUON[1]) * A + _f32(MUON[2]) * (A @ A)) @ X
        want = 0.5 * (X if m <= n else X.T)
        tol = ref.orthogonalize_bound(norms, [MUON] * 5, 0.5, m * n) + 1.01 * ref.HALF_STEP[dtype] * float(torch.linalg.vector_norm(want))
        err = float(torch.linalg.vector_norm(out[i].double() - want))
        assert err <= tol, (i, err, tol)


def test_orthogonalize_gives_singular_values_near_one():
    """And the same singular vectors: U' out V is the diagonal of the mapped singular values."""
    G = _gradient(200, 300, 77)
    U, s, Vt = np.linalg.svd(np.float32(G).astype(np.float64), full_matrices=False)
    got = _check_ortho(G[None], "f32", steps=12, coefficients=CUBIC)[0]
    D = U.T @ got @ Vt.T
    x = s / np.linalg.norm(s)
    for _ in range(12):
        x = 1.5 * x - 0.5 * x ** 3
    assert np.abs(D - np.diag(x)).max() <= 1.5 ** 12 * 12 * 4 * 2.0 ** -22 and (x[:100] > 0.9).all()


def test_orthogonalize_of_many_small_matrices():
    """More matrices than the work space takes at once; a batch gives what its matrices give alone."""
    import torch
    from paper_2510_02470_amd.binding import orthogonalize

    g = torch.Generator(device="cuda").manual_seed(3)
    G = torch.randn(7000, 9, 40, generator=g, device="cuda")
    out = orthogonalize(G)
    for i in (0, 1, 2499, 4000, 6999):
        assert torch.equal(out[i], orthogonalize(G[i]))
    A = out @ out.transpose(1, 2).contiguous()
    ev = torch.linalg.eigvalsh(A[:200].cpu())
    assert float(ev.max()) < 1.3 ** 2 and float(ev.min()) > 0.6 ** 2


# ---- together, and in the ways programs call --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_from_logits_to_the_update_of_the_kept_rows(dtype):
    """Labels drawn from a head's own logits, the errors as factors of its rows, a selection by them, and the kept rows' gradient made
    an update."""
    import torch
    from paper_2510_02470_amd.binding import Sage, logit_error, orthogonalize, sample

    N, C, dh, ell = 640, 40, 64, 32
    td = _tdtype(dtype)
    g = torch.Generator(device="cuda").manual_seed(6)
    H = torch.relu(torch.randn(N, dh, generator=g, device="cuda")).to(td)
    W = torch.randn(C, dh, generator=g, device="cuda") / 4
    z = (H.float() @ W.T).to(td)
    u = torch.rand(N, generator=g, device="cuda")
    y, logp = sample(z, u)
    E, loss = logit_error(z, y)
    assert bool(((loss + logp).abs() <= 2.0 ** -18 * (1 + loss)).all())  # at temperature 1 the loss is -logp
    zh = z.double().cpu().numpy()
    want, want_loss, _ = ref.logit_error(zh, y.cpu().numpy(), np.ones(N))
    assert np.abs(E.double().cpu().numpy() - want).max() <= ref.HALF_STEP[dtype] + 40 * 2.0 ** -24
    rows = (E.float()[:, :, None] * H.float()[:, None, :]).reshape(N, C * dh)
    G = torch.cat([rows, E.float()], 1).to(td).contiguous()

    def pick(update, score):
        s = Sage(ell, C * (dh + 1), dtype=dtype, max_rows=N)
        for lo in range(0, N, 128):
            update(s, slice(lo, lo + 128))
        s.fd_basis(16)
        for lo in range(0, N, 128):
            score(s, slice(lo, lo + 128))
        idx, sketch = s.select(0.25), s.sketch()
        s.close()
        return idx, sketch

    idx, sketch = pick(lambda s, b: s.fd_update_outer(E[b].contiguous(), H[b].contiguous()),
                       lambda s, b: s.score_outer(E[b].contiguous(), H[b].contiguous()))
    _, by_rows = pick(lambda s, b: s.fd_update(G[b]), lambda s, b: s.score(G[b]))
    assert torch.equal(sketch, by_rows) and len(idx) == N // 4
    grad = (E[idx].float().T @ H[idx].float()).to(td)
    out = orthogonalize(grad, scale=0.2)
    ref_out, norms = ref.orthogonalize(grad.double().cpu().numpy(), [[_f32(v) for v in MUON]] * 5, _f32(1e-7), _f32(0.2))
    err = np.linalg.norm(out.double().cpu().numpy() - ref_out)
    assert err <= ref.orthogonalize_bound(norms, [MUON] * 5, 0.2, C * dh) + 1.01 * ref.HALF_STEP[dtype] * np.linalg.norm(ref_out)


def test_captured_and_replayed_on_other_data():
    import torch
    from paper_2510_02470_amd.binding import logit_error, orthogonalize, sample

    g = torch.Generator(device="cuda").manual_seed(1)

    def fresh():
        return (3 * torch.randn(6, 40_000, generator=g, device="cuda"), torch.rand(6, generator=g, device="cuda"),
                torch.randn(2, 90, 130, generator=g, device="cuda"), torch.randn(300, 200, generator=g, device="cuda").bfloat16())

    z, u, G, B = fresh()

    def step():
        y, logp = sample(z, u, temperature=0.8, top_k=100, top_p=0.9)
        E, loss = logit_error(z, y)
        return y, logp, E, loss, orthogonalize(G), orthogonalize(B, scale=2.0)

    step()
    graphs = []
    for _ in range(2):  # two graphs have their own work space
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, step()))
        graphs[-1] = (graph, graphs[-1][1])
    for i in range(5):
        for t, v in zip((z, u, G, B), fresh()):
            t.copy_(v)
        graphs[i % 2][0].replay()
        if i > 2:
            graphs[(i + 1) % 2][0].replay()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(graphs[i % 2][1], want):
            assert torch.equal(a, b)


def test_on_another_stream():
    import torch
    from paper_2510_02470_amd.binding import logit_error, orthogonalize, sample

    z = 2 * torch.randn(64, 5000, device="cuda")
    u = torch.rand(64, device="cuda")
    G = torch.randn(150, 260, device="cuda")
    y, logp = sample(z, u, top_p=0.9)
    E, loss = logit_error(z, y)
    O = orthogonalize(G)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        z2 = torch.zeros_like(z)
        torch.cuda._sleep(2_000_000)
        z2.copy_(z)
        y2, logp2 = sample(z2, u, top_p=0.9)
        E2, loss2 = logit_error(z2, y2)
        O2 = orthogonalize(G)
    side.synchronize()
    for a, b in zip((y, logp, E, loss, O), (y2, logp2, E2, loss2, O2)):
        assert torch.equal(a, b)


def test_no_rows():
    import torch
    from paper_2510_02470_amd.binding import logit_error, orthogonalize, sample

    z = torch.empty(0, 12, device="cuda")
    y, logp = sample(z, torch.empty(0, device="cuda"))
    E, loss = logit_error(z, y)
    assert y.shape == logp.shape == loss.shape == (0,) and E.shape == (0, 12)
    assert orthogonalize(torch.empty(0, 3, 4, device="cuda")).shape == (0, 3, 4)


def test_binding_refusals():
    import torch
    from paper_2510_02470_amd.binding import SageError, logit_error, orthogonalize, sample

    z, u = torch.zeros(4, 6, device="cuda"), torch.zeros(4, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    G = torch.randn(3, 5, 7, device="cuda")
    for call in (
        lambda: sample(z.double(), u), lambda: sample(z.T, u), lambda: sample(z[None], u), lambda: sample(z, u[:3]), lambda: sample(z, u.double()),
        lambda: sample(z, u.cpu()), lambda: sample(z, u, temperature=torch.ones(3, device="cuda")),
        lambda: sample(z, u, top_k=torch.ones(4, device="cuda")), lambda: sample(z[:, :0], u), lambda: sample(z[:1].expand(4, 6), u),
        lambda: logit_error(z, y.long()), lambda: logit_error(z, y[:2]), lambda: logit_error(z, y, weights=u.half()),
        lambda: logit_error(z, y, out=z[:, :5]), lambda: logit_error(z, y, out=z.view(torch.int32)), lambda: logit_error(z, y, dtype=torch.float16),
        lambda: logit_error(z, y, out=z, dtype=torch.bfloat16),
        lambda: orthogonalize(G.half()), lambda: orthogonalize(G[:, ::2, ::2]), lambda: orthogonalize(G, out=G.transpose(1, 2)),
        lambda: orthogonalize(G, out=torch.empty(3, 7, 5, device="cuda").transpose(1, 2)), lambda: orthogonalize(G[0, 0]),
        lambda: orthogonalize(G, steps=0), lambda: orthogonalize(G, steps=3, coefficients=[MUON] * 2), lambda: orthogonalize(G[:1].expand(3, 5, 7)),
        lambda: orthogonalize(G, out=G.bfloat16()), lambda: orthogonalize(G, eps=-1.0),
    ):
        with pytest.raises(SageError):
            call()
