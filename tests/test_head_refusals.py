"""What sage_sample, sage_logit_error and sage_orthogonalize refuse, through the C ABI: no call here reaches a GPU."""
import ctypes as C

import pytest

from paper_2510_02470_amd import binding
from paper_2510_02470_amd.binding import SAGE_BF16, SAGE_ERR_ARG, SAGE_F32, SAGE_OK

MEM = (C.c_char * 8192)()
P = (C.addressof(MEM) + 255) // 256 * 256  # an aligned address that nothing reads


@pytest.mark.parametrize("change", [
    {"logits": 0}, {"logits": P + 2}, {"dtype": 2}, {"dtype": -1}, {"rows": -1}, {"classes": 0}, {"classes": binding.MAX_CLASSES + 1, "ld": 1 << 21},
    {"ld": 9}, {"u": 0}, {"labels": 0}, {"ld": 1 << 60}, {"rows": 1 << 40, "ld": 1 << 30}])
def test_sample_refuses(change):
    a = dict(logits=P, dtype=SAGE_F32, rows=2, classes=10, ld=10, u=P, labels=P)
    a.update(change)
    L = binding.lib()
    how = binding.SageSampling(1.0, 0, 1.0, 0.0)
    assert L.sage_sample(a["logits"], a["dtype"], a["rows"], a["classes"], a["ld"], a["u"], C.byref(how), a["labels"], None, None) == SAGE_ERR_ARG


@pytest.mark.parametrize("change", [
    {"logits": 0}, {"logits": P + 1, "dtype": SAGE_BF16}, {"dtype": 5}, {"rows": -3}, {"classes": 0}, {"ld": 9}, {"labels": 0}, {"e_dtype": 7},
    {"ld_e": 9}, {"E": P + 4096 + 2}, {"E": P + 4}, {"E": P, "e_dtype": SAGE_BF16}, {"E": P, "ld_e": 11}, {"E": P + 76}])
def test_logit_error_refuses(change):
    a = dict(logits=P, dtype=SAGE_F32, rows=2, classes=10, ld=10, labels=P, E=P + 4096, e_dtype=SAGE_F32, ld_e=10)
    a.update(change)
    L = binding.lib()
    assert L.sage_logit_error(a["logits"], a["dtype"], a["rows"], a["classes"], a["ld"], a["labels"], None, a["E"], a["e_dtype"], a["ld_e"],
                              None, None) == SAGE_ERR_ARG


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change", [
    {"G": 0}, {"G": P + 2}, {"out": 0}, {"out": P + 4096 + 2}, {"dtype": 2}, {"batch": -1}, {"rows": 0}, {"cols": 0}, {"rows": 32769}, {"cols": 40000, "ld": 40000},
    {"ld": 4}, {"ld_out": 4}, {"stride": 14}, {"stride_out": 14}, {"steps": 0}, {"steps": 33}, {"eps": -1e-9}, {"eps": NAN}, {"eps": INF},
    {"scale": NAN}, {"scale": INF}, {"coef": None}, {"coef": (NAN, 0, 0)}, {"coef": (INF, 0, 0)}, {"coef": (0, 0, 2000.0)},
    {"coef": (40.0, 0, 0)},  # 40 * 40: singular values would pass 2^10
    {"coef": (900.0, 900.0, 900.0)}, {"out": P + 4}, {"out": P, "ld_out": 6, "stride_out": 18}, {"work": 0}, {"work": P + 8}, {"work_bytes": 10}])
def test_orthogonalize_refuses(change):
    a = dict(G=P, dtype=SAGE_F32, batch=2, rows=3, cols=5, ld=5, stride=15, coef=binding.MUON, steps=2, eps=1e-7, scale=1.0, out=P + 4096, ld_out=5,
             stride_out=15, work=P, work_bytes=1 << 40)
    a.update(change)
    L = binding.lib()
    coef = None if a["coef"] is None else (C.c_float * 99)(*(tuple(a["coef"]) * 33))
    assert L.sage_orthogonalize(a["G"], a["dtype"], a["batch"], a["rows"], a["cols"], a["ld"], a["stride"], coef, a["steps"], a["eps"], a["scale"],
                                a["out"], a["ld_out"], a["stride_out"], a["work"], a["work_bytes"], None) == SAGE_ERR_ARG


def test_work_space_sizes():
    L = binding.lib()
    n = C.c_size_t(1)
    assert L.sage_orthogonalize_work(SAGE_F32, 0, 3, 5, C.byref(n)) == SAGE_OK and n.value == 0
    assert L.sage_orthogonalize_work(SAGE_F32, 1, 3, 5, None) == SAGE_ERR_ARG
    assert L.sage_orthogonalize_work(3, 1, 3, 5, C.byref(n)) == SAGE_ERR_ARG
    assert L.sage_orthogonalize_work(SAGE_F32, 1, 0, 5, C.byref(n)) == SAGE_ERR_ARG
    sizes = []
    for batch in (1, 100, 100_000, 1_000_000):
        assert L.sage_orthogonalize_work(SAGE_BF16, batch, 200, 300, C.byref(n)) == SAGE_OK
        sizes.append(n.value)
    assert 0 < sizes[0] < sizes[1] <= sizes[2] == sizes[3] <= 1 << 30  # many matrices are taken in turns
    assert L.sage_orthogonalize_work(SAGE_F32, 1, 32768, 32768, C.byref(n)) == SAGE_OK and n.value < 64 << 30


def test_nothing_to_do_is_no_error():
    L = binding.lib()
    assert L.sage_sample(None, SAGE_F32, 0, 10, 10, None, None, None, None, None) == SAGE_OK
    assert L.sage_logit_error(None, SAGE_F32, 0, 10, 10, None, None, None, SAGE_F32, 10, None, None) == SAGE_OK
    assert L.sage_logit_error(P, SAGE_F32, 2, 10, 10, P, None, None, SAGE_F32, 10, None, None) == SAGE_OK  # neither E nor loss
    coef = (C.c_float * 3)(*binding.MUON)
    assert L.sage_orthogonalize(None, SAGE_F32, 0, 3, 5, 5, 15, coef, 1, 0.0, 1.0, None, 5, 15, None, 0, None) == SAGE_OK


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch

    z, u, y = torch.zeros(2, 5), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: binding.sample(z, u), lambda: binding.logit_error(z, y), lambda: binding.orthogonalize(z),
                 lambda: binding.orthogonalize(z, steps=2, coefficients=[(1.0, 0.0, 0.0)]),
                 lambda: binding.orthogonalize(z, coefficients=(1.0, 2.0))):
        with pytest.raises(binding.SageError) as e:
            call()
        assert e.value.code == SAGE_ERR_ARG


def test_polynomials_are_bounded_over_the_whole_interval():
    """The bound that scales the parts is that of the polynomial's extremes, inside the interval or at its ends: coefficients just
    inside and just outside of what is taken."""
    L = binding.lib()

    def rc(*triples):
        coef = (C.c_float * (3 * len(triples)))(*[v for t in triples for v in t])
        return L.sage_orthogonalize(None, SAGE_F32, 0, 1, 1, 1, 1, coef, len(triples), 0.0, 1.0, None, 1, 1, None, 0, None)

    assert rc((1000.0, 0, 0)) == SAGE_OK and rc((1024.0, 0, 0)) == SAGE_ERR_ARG
    # 600 s - 600 s^3 vanishes at both ends and is 231 in between; then times 4, and times 5
    assert rc((600.0, -600.0, 0), (4.0, 0, 0)) == SAGE_OK
    assert rc((600.0, -600.0, 0), (5.0, 0, 0)) == SAGE_ERR_ARG
    assert rc(*[binding.MUON] * 32) == SAGE_OK  # stays where it is
    assert rc(*[(1.5, -0.5, 0.0)] * 32) == SAGE_OK
