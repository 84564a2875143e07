"""sample, logit_error and orthogonalize where layouts, settings and values meet that each alone are ordinary."""
import math

import numpy as np
import pytest

import head_reference as ref
from test_gpu_head import MUON, _f32, _tdtype

pytestmark = pytest.mark.gpu


# ---- orthogonalize ----------------------------------------------------------------------------------------------

def _wide(t, step, fill):
    """The same single row or column (or several), its elements `step` apart in memory that holds `fill`; and that memory."""
    import torch

    n, b = max(t.shape[-2:]), t.shape[0]
    hold = torch.full((b, n * step + 3), fill, dtype=t.dtype, device="cuda")
    view = hold[:, :n * step:step]
    view = view[:, None, :] if t.shape[1] == 1 else view[:, :, None]
    view.copy_(t)
    return view, hold


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 100), (4, 1, 100), (4, 100, 1), (2, 1, 700)])
def test_single_rows_whose_elements_are_apart(shape, dtype):
    """What lies between the elements is not read, and left as it was."""
    import torch
    from paper_2510_02470_amd.binding import orthogonalize

    g = torch.Generator(device="cuda").manual_seed(shape[-1])
    G = torch.randn(shape, generator=g, device="cuda").to(_tdtype(dtype))
    want = torch.stack([torch.from_numpy(ref.orthogonalize(x.double().cpu().numpy(), [[_f32(v) for v in MUON]] * 5, _f32(1e-7), 1.0)[0]) for x in G])
    # a matrix of rank one: one singular value, of at most 1.25 after each step
    tol = ref.orthogonalize_bound([1.0] * 5, [MUON] * 5, 1.0, G[0].numel()) + 1.01 * ref.HALF_STEP[dtype] * 1.25
    for step, out_step in ((5, None), (5, 1), (1, 3), (2, 4), (1, 1)):
        given, _ = _wide(G, step, math.nan)
        out = hold = None
        if out_step:
            out, hold = _wide(torch.zeros_like(G), out_step, 7.0)
        res = orthogonalize(given, out=out)
        assert res.shape == G.shape and (out is None or res.data_ptr() == out.data_ptr())
        assert float(torch.linalg.vector_norm(res.double().cpu() - want, dim=(1, 2)).max()) <= tol
        if out_step:
            assert int((hold == 7.0).sum()) == hold.numel() - G.numel()


# ---- sample -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("C", [33_001, 131_072])
def test_long_rows_by_value_and_by_class_have_the_same_labels(C):
    """bf16 rows, of whose values the weights are found by value, and the same rows as fp32, where every class is looked at: the border of
    top-p moves with the sum of the values near zero, which work-groups add up on their own just before. All rows, again and again."""
    import torch
    from paper_2510_02470_amd.binding import sample

    g = torch.Generator(device="cuda").manual_seed(C)
    n = 600
    z = 1.5 * torch.randn(n, C, generator=g, device="cuda") - 3.0
    near = torch.randint(0, C, (n, 800), generator=g, device="cuda")
    z.scatter_(1, near, 0.001 * torch.randn(n, 800, generator=g, device="cuda"))
    z.scatter_(1, torch.randint(0, C, (n, 6), generator=g, device="cuda"), 2.0)
    z = z.bfloat16()
    wide = z.float()
    u = torch.rand(n, generator=g, device="cuda")
    p = torch.rand(n, generator=g, device="cuda")
    for T in (1.0, 0.4):
        want = sample(wide, u, temperature=T, top_p=p)
        for _ in range(10):
            labels, logp = sample(z, u, temperature=T, top_p=p)
            assert torch.equal(labels, want[0]) and torch.equal(logp, want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(6, 1), (6, 5), (8, 700), (8, 9001), (8, 40_000), (260, 33_001)])
def test_min_p_of_one_at_any_temperature(n, C, dtype):
    """What is left are the classes equal to the greatest, of those that the other settings leave; at an infinite temperature too,
    where all classes that are not masked have the same weight."""
    import torch
    from paper_2510_02470_amd.binding import sample

    rng = np.random.default_rng(C)
    z = 2.0 * rng.standard_normal((n, C))
    z[rng.random(z.shape) < 0.3] = -np.inf
    z[:, C // 2] = 1.0
    z[1] = np.round(z[1])  # several greatest
    z[2] = 0.25
    z[3] = np.where(np.arange(C) % 3 == 1, 9.0, z[3])
    z[4] = -np.inf
    z[4, C - 1] = -5.0
    zd = torch.from_numpy(z).cuda().to(_tdtype(dtype))
    zh = zd.double().cpu().numpy()
    u = rng.random(n, dtype=np.float32)
    ud = torch.from_numpy(u).cuda()
    for T in (math.inf, 1.0, 1e30):
        for k, p in ((0, 1.0), (3, 1.0), (0, 0.6), (3, 0.5), (max(1, 2 * C // 3), 0.9)):
            for m in (1.0, 2.0, math.inf):
                labels, logp = (t.cpu().numpy() for t in sample(zd, ud, temperature=T, top_k=k, top_p=p, min_p=m))
                for i in range(n if n < 100 else 12):
                    kept, w = ref.kept_classes(zh[i], T, k, _f32(p), 0.0)
                    kept = kept[zh[i, kept] == zh[i].max()]
                    c = np.cumsum(w[kept])
                    j = kept[np.searchsorted(c, min(int(float(u[i]) * float(c[-1])), int(c[-1]) - 1), side="right")]
                    assert labels[i] == j, (T, k, p, m, i, labels[i], j)
                    assert abs(logp[i] + math.log(len(kept))) <= 2.0 ** -24 * math.log(len(kept)) + 1e-12
    # as one request among others
    per_row = lambda values: torch.from_numpy(np.resize(np.float32(values), n)).cuda()
    T, m = np.resize(np.float32([math.inf, 1.0, math.inf, 0.7]), n), np.resize(np.float32([1.0, 0.1, 0.1]), n)
    labels, _ = sample(zd, ud, temperature=per_row([math.inf, 1.0, math.inf, 0.7]), min_p=per_row([1.0, 0.1, 0.1]))
    for i, j in enumerate(labels.cpu().numpy()):
        if T[i] < math.inf or m[i] < 1:
            assert j == ref.sample_row(zh[i], float(u[i]), float(T[i]), 0, 1.0, float(m[i]))[0]
        else:
            assert zh[i, j] == zh[i].max()


# ---- logit_error ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(3000, 2), (40, 1000), (5, 9001), (300, 40_000), (3, 140_001), (260, 90_001)])
def test_losses_do_not_depend_on_the_type_of_the_errors(n, C, dtype):
    import ctypes

    import torch
    from paper_2510_02470_amd import binding

    g = torch.Generator(device="cuda").manual_seed(C)
    z = (3 * torch.randn(n, C, generator=g, device="cuda")).to(_tdtype(dtype))
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.where(torch.arange(n, device="cuda") % 2 == 0, z.float().argmax(1).int(), y)
    wide = binding.logit_error(z, y, dtype=torch.float32)[1]
    narrow = binding.logit_error(z, y, dtype=torch.bfloat16)[1]
    assert torch.equal(wide, narrow)
    alone = torch.zeros_like(wide)
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    code = binding.SAGE_BF16 if dtype == "bf16" else binding.SAGE_F32
    for e_code in (binding.SAGE_F32, binding.SAGE_BF16):
        rc = binding.lib().sage_logit_error(p(z), code, n, C, C, p(y), None, None, e_code, C, p(alone), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == binding.SAGE_OK and torch.equal(alone, wide)
        alone.zero_()


def test_losses_of_learnt_examples_with_one_rival():
    """log1p(e^-d): d is exact, the exponential is off by an ulp (2^-23) of the power of two and half of one (2^-24) of what is added to it for
    the rest of the product d log2 e, and the loss is rounded once (2^-24): four half steps, and one for the products of these."""
    import torch
    from paper_2510_02470_amd.binding import logit_error

    for shift in (0.0, 3.0, -40.0):
        z = torch.zeros(4000, 2, device="cuda", dtype=torch.bfloat16)
        z[:, 0] = shift
        z[:, 1] = shift - torch.linspace(0.05, 80.0, 4000, device="cuda")
        d = (z[:, 0].double() - z[:, 1].double())
        want = torch.log1p(torch.exp(-d))
        for dtype in (torch.bfloat16, torch.float32):
            _, loss = logit_error(z, torch.zeros(4000, device="cuda", dtype=torch.int32), dtype=dtype)
            err = (loss.double() - want).abs() / want
            assert float(err.max()) <= 5 * 2.0 ** -24, (dtype, shift, float(err.max()))


# ---- orthogonalize: coefficients --------------------------------------------------------------------------------

@pytest.mark.parametrize("m,n", [(24, 40), (150, 140)])
def test_nearly_cubic_coefficients(m, n):
    """Singular values stretched past the extreme of the next step's polynomial, whose fifth power is as good as none."""
    import torch
    from paper_2510_02470_amd.binding import orthogonalize

    g = torch.Generator(device="cuda").manual_seed(m)
    Q = torch.linalg.qr(torch.randn(m, m, generator=g, device="cuda", dtype=torch.float64).cpu())[0]
    G = torch.zeros(m, n, dtype=torch.float64)
    k = min(m, n, 20)
    G[:, :k] = Q[:, :k] * torch.linspace(0.05, 1.0, k, dtype=torch.float64)
    G = G.float()
    # the bound of the first step's singular values is 1.732, where 1.5 s - 0.5 s^3 is next to 0; at 1 it is 1
    triples = [(1.7287, 0.0, 0.0), (1.5, -0.5, 1e-30), (1.5, -0.5, -1e-25)]
    out = orthogonalize(G.cuda(), steps=3, coefficients=triples, eps=0.0).double().cpu().numpy()
    want, norms = ref.orthogonalize(G.double().numpy(), [[_f32(v) for v in t] for t in triples], 0.0, 1.0)
    # singular values up to 1.73: slopes up to 3, the terms' sum at most 1.5 * 1.73 + 0.5 * 1.73^3 = 5.2
    tol = ref.orthogonalize_bound(norms, [(3.0, -1.1, 0.0)] * 3, 1.0, m * n)
    assert np.linalg.norm(out - want) <= tol


# ---- outputs between the rows of the inputs ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(1, 9), (5, 40), (300, 1001), (4, 70_001), (2, 140_000)])
def test_errors_beside_their_logits(n, C, dtype):
    """Columns of one buffer: what is before, between and behind them stays as it was."""
    import torch
    from paper_2510_02470_amd.binding import SageError, logit_error

    g = torch.Generator(device="cuda").manual_seed(C)
    z = (3 * torch.randn(n, C, generator=g, device="cuda")).to(_tdtype(dtype))
    y = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    want, want_loss = logit_error(z, y)
    for first, second in ((3, C + 3), (C + 9, 4)):
        buf = torch.full((n, 2 * C + 20), 7.0, dtype=z.dtype, device="cuda")
        logits, E = buf[:, first:first + C], buf[:, second:second + C]
        logits.copy_(z)
        loss = logit_error(logits, y, out=E)[1]
        assert torch.equal(E, want) and torch.equal(loss, want_loss) and torch.equal(logits, z)
        E.fill_(7.0)
        logits.fill_(7.0)
        assert bool((buf == 7.0).all())
        for shift in (-1, 1, C - 1, 1 - C):
            if n > 1 and 0 <= first + shift:
                with pytest.raises(SageError):
                    logit_error(logits, y, out=buf[:, first + shift:first + shift + C])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,m,n", [(1, 5, 9), (3, 130, 70), (2, 64, 200), (1, 1, 30)])
def test_updates_beside_their_gradients(b, m, n, dtype):
    import torch
    from paper_2510_02470_amd.binding import SageError, orthogonalize

    g = torch.Generator(device="cuda").manual_seed(n)
    G = torch.randn(b, m, n, generator=g, device="cuda").to(_tdtype(dtype))
    want = orthogonalize(G)
    for first, second in ((2, n + 2), (n + 7, 3)):
        buf = torch.full((b, m + 1, 2 * n + 10), 7.0, dtype=G.dtype, device="cuda")
        given, out = buf[:, :m, first:first + n], buf[:, :m, second:second + n]
        given.copy_(G)
        orthogonalize(given, out=out)
        assert torch.equal(out, want) and torch.equal(given, G)
        out.fill_(7.0)
        given.fill_(7.0)
        assert bool((buf == 7.0).all())
        with pytest.raises(SageError):
            orthogonalize(given, out=buf[:, :m, first + 1:first + 1 + n])
        if m > 1:
            with pytest.raises(SageError):
                orthogonalize(given, out=buf[:, 1:, first:first + n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,b,n", [(40, 3, 17), (130, 4, 70), (70, 5, 130), (9, 6, 1)])
def test_matrices_side_by_side(m, b, n, dtype):
    """The column slices of one matrix, as a batch: from and to such, in place, and with the result between the slices."""
    import ctypes

    import torch
    from paper_2510_02470_amd import binding
    from paper_2510_02470_amd.binding import SageError, orthogonalize

    g = torch.Generator(device="cuda").manual_seed(n)
    G = torch.randn(b, m, n, generator=g, device="cuda").to(_tdtype(dtype))
    want = orthogonalize(G)

    def slices(cols):
        W = torch.full((m + 1, b * cols + 3), 7.0, dtype=G.dtype, device="cuda")
        return W, W.as_strided((b, m, cols), (cols, W.stride(0), 1))

    W, given = slices(n)
    V, out = slices(n)
    given.copy_(G)
    assert torch.equal(orthogonalize(given), want)
    assert torch.equal(orthogonalize(G, out=out), want) and torch.equal(orthogonalize(given, out=out), want) and torch.equal(given, G)
    assert int((V == 7.0).sum()) >= V.numel() - G.numel()
    out.fill_(7.0)
    assert bool((V == 7.0).all())
    turned = orthogonalize(given.transpose(1, 2))
    assert torch.equal(turned, want.transpose(1, 2))
    # one slice with the next one's place for its result
    W, pairs = slices(2 * n)
    pairs[:, :, :n].copy_(G)
    orthogonalize(pairs[:, :, :n], out=pairs[:, :, n:])
    assert torch.equal(pairs[:, :, n:], want) and torch.equal(pairs[:, :, :n], G)
    if n > 1:
        with pytest.raises(SageError):
            orthogonalize(pairs[:, :, :n], out=pairs[:, :, n - 1:2 * n - 1])
    orthogonalize(pairs[:, :, :n], out=pairs[:, :, :n])
    assert torch.equal(pairs[:, :, :n], want)
    pairs.fill_(7.0)
    assert bool((W == 7.0).all())
    # the library's own check of matrices with elements in common
    L, st = binding.lib(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    code = binding.SAGE_BF16 if dtype == "bf16" else binding.SAGE_F32
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    coef = (ctypes.c_float * 3)(*MUON)
    res = torch.empty_like(G)
    for ld, stride in ((b * n, n - 1), (b * n - 1, n)):
        assert L.sage_orthogonalize(p(G), code, b, m, n, ld, stride, coef, 1, 0.0, 1.0, p(res), n, m * n, p(work), work.numel(), st) == binding.SAGE_ERR_ARG


# ---- more matrices than the work space takes at once ------------------------------------------------------------

@pytest.mark.parametrize("b,m,n,dtype,pad", [(2400, 1, 513, "f32", 0), (2300, 20, 520, "bf16", 3), (900, 129, 129, "f32", 0), (900, 150, 129, "bf16", 1)])
def test_batches_in_several_turns(b, m, n, dtype, pad):
    """Every matrix, the last turn's fewer ones among them, against 64-bit products; what lies between the matrices stays as it was."""
    import ctypes

    import torch
    from paper_2510_02470_amd import binding

    code, need = binding.SAGE_BF16 if dtype == "bf16" else binding.SAGE_F32, ctypes.c_size_t(0)
    sizes = []
    for count in (b, 2 * b):
        assert binding.lib().sage_orthogonalize_work(code, count, m, n, ctypes.byref(need)) == binding.SAGE_OK
        sizes.append(need.value)
    assert sizes[0] == sizes[1]  # (a turn does not take them all)
    g = torch.Generator(device="cuda").manual_seed(b + m)
    G = torch.randn(b, m + pad, n + pad, generator=g, device="cuda").to(_tdtype(dtype))[:, :m, :n]
    hold = torch.full((b, m + 2 * pad, n + pad), 7.0, dtype=G.dtype, device="cuda")
    out = hold[:, :m, :n]
    binding.orthogonalize(G, out=out)
    X = G.double() if m <= n else G.double().transpose(1, 2).contiguous()
    X = X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + _f32(1e-7))
    norms = []
    for _ in range(5):
        norms.append(float(torch.linalg.vector_norm(X, dim=(1, 2)).max()))
        A = X @ X.transpose(1, 2).contiguous()
        X = _f32(MUON[0]) * X + (_f32(MUON[1]) * A + _f32(MUON[2]) * (A @ A)) @ X
    want = X if m <= n else X.transpose(1, 2)
    size = torch.linalg.vector_norm(want, dim=(1, 2))
    tol = ref.orthogonalize_bound(norms, [MUON] * 5, 1.0, m * n) + 1.01 * ref.HALF_STEP[dtype] * size
    err = torch.linalg.vector_norm(out.double() - want, dim=(1, 2))
    assert bool((err <= tol).all()), (int((err > tol).nonzero()[0]), float((err / tol).max()))
    out.fill_(7.0)
    assert bool((hold == 7.0).all())
