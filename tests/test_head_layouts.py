"""Where sage_orthogonalize is told to read and write for matrices of every layout: the calls are recorded and compared with the
tensors' own addresses. No GPU."""
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2510_02470_amd import binding


class Recorder:
    """In the library's place: keeps what a call of sage_orthogonalize was given."""

    def sage_orthogonalize_work(self, code, batch, rows, cols, need):
        need._obj.value = 256
        return binding.SAGE_OK

    def sage_orthogonalize(self, G, code, batch, rows, cols, ld, stride, coef, steps, eps, scale, out, ld_out, stride_out, *rest):
        self.sizes, self.G, self.out = (batch, rows, cols), (G, ld, stride), (out, ld_out, stride_out)
        return binding.SAGE_OK

    def sage_strerror(self, code):
        return b"refused"


@pytest.fixture
def recorder(monkeypatch):
    r, empty = Recorder(), torch.empty
    monkeypatch.setattr(binding, "lib", lambda: r)
    monkeypatch.setattr(binding, "_device", lambda torch, t, what: t.get_device())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k))
    return r


def _elements(sizes, place):
    """Addresses that the library takes for (matrix, row, column), in its order."""
    (batch, rows, cols), (base, ld, stride) = sizes, place
    i, r, t = np.ogrid[:batch, :rows, :cols]
    return base + 4 * (i * stride + r * ld + t)


def _addresses(t):
    t = t[None] if t.dim() == 2 else t
    i, r, c = np.ogrid[:t.shape[0], :t.shape[1], :t.shape[2]]
    return t.data_ptr() + 4 * (i * t.stride(0) + r * t.stride(1) + c * t.stride(2))


def _check(r, G, out):
    res = binding.orthogonalize(G, out=out)
    assert out is None or res is out
    assert res.shape == G.shape
    g, o, at_g, at_o = _addresses(G), _addresses(res), _elements(r.sizes, r.G), _elements(r.sizes, r.out)
    same = at_g.shape == g.shape and np.array_equal(at_g, g) and np.array_equal(at_o, o)
    turned = at_g.shape == g.transpose(0, 2, 1).shape and np.array_equal(at_g.transpose(0, 2, 1), g) and np.array_equal(at_o.transpose(0, 2, 1), o)
    assert same or turned, (r.sizes, r.G, r.out)


def _line(shape, step, batch_step=None):
    """A matrix (or several) of one row or one column, its elements `step` apart."""
    n = max(shape[-2:])
    batch = shape[0] if len(shape) == 3 else 1
    batch_step = n * step + 3 if batch_step is None else batch_step
    t = torch.zeros(batch * batch_step + n * step)
    long = (step, 0) if shape[-2] == n else (0, step)
    long = tuple(s or 7 for s in long)  # (the stride of a side of one has no meaning)
    return t.as_strided(shape, ((batch_step,) if len(shape) == 3 else ()) + long)


@pytest.mark.parametrize("shape", [(1, 100), (100, 1), (4, 1, 100), (4, 100, 1), (1, 1), (1, 1, 1), (1, 1, 50)])
@pytest.mark.parametrize("step", [1, 2, 5])
@pytest.mark.parametrize("out_step", [None, 1, 2, 5, 101])
def test_single_rows_and_columns(recorder, shape, step, out_step):
    _check(recorder, _line(shape, step), None if out_step is None else _line(shape, out_step))


def test_single_rows_as_programs_have_them(recorder):
    W, buf = torch.zeros(100, 5), torch.zeros(100, 130)
    _check(recorder, W[:, :1].T, None)
    _check(recorder, W[:, :1].T, torch.zeros(1, 100))
    _check(recorder, torch.zeros(1, 100), buf[:, :1].T)
    _check(recorder, W[:, 2:3], buf[:, 3:4])
    _check(recorder, W[3:4], None)
    _check(recorder, W[3:4], W[3:4])
    _check(recorder, torch.zeros(4, 100, 5)[:, :, :1].transpose(1, 2), torch.zeros(4, 1, 100))


def test_matrices(recorder):
    for G, out in ((torch.zeros(6, 9), None), (torch.zeros(9, 6).T, None), (torch.zeros(8, 12)[:6, :9], torch.zeros(6, 9)),
                   (torch.zeros(9, 6).T, torch.zeros(10, 7)[:9, :6].T), (torch.zeros(3, 7, 10)[:, :6, :9], None),
                   (torch.zeros(3, 9, 6).transpose(1, 2), None), (torch.zeros(3, 9, 6).transpose(1, 2), torch.zeros(5, 9, 8)[1:4, :, :6].transpose(1, 2))):
        _check(recorder, G, out)


def test_refused_layouts(recorder):
    G = torch.zeros(6, 9)
    for G, out in ((G, torch.zeros(9, 6).T), (torch.zeros(9, 6).T, G), (torch.zeros(6, 18)[:, ::2], None), (torch.zeros(1, 9).expand(6, 9), None),
                   (torch.zeros(6, 1).expand(6, 9), None), (torch.zeros(1, 1).expand(1, 9), None), (torch.zeros(1, 9).expand(2, 1, 9), None),
                   (torch.zeros(1, 9), torch.zeros(1, 1).expand(1, 9))):
        with pytest.raises(binding.SageError):
            binding.orthogonalize(G, out=out)


def test_common_elements_of_rows(tmp_path):
    """rows_meet_check.cc; and the check itself: it must refuse a comparison of the spans."""
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "rows_meet_check")
    csrc = os.path.join(os.path.dirname(here), "paper_2510_02470_amd", "csrc")
    b = subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", csrc, os.path.join(here, "rows_meet_check.cc"), "-o", exe],
                       capture_output=True, text=True)
    assert b.returncode == 0, b.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "rows_meet_check ok" in r.stdout, r.stdout
    assert subprocess.run([exe, "spans"], capture_output=True, text=True, timeout=120).returncode == 1


def _heads(rows, heads, cols, pad=0):
    """The column slices of one matrix, as a batch."""
    return torch.zeros(rows, heads * cols + pad)[:, :heads * cols].view(rows, heads, cols).transpose(0, 1)


def test_matrices_side_by_side(recorder):
    for G, out in ((_heads(6, 4, 9), None), (_heads(6, 4, 9), torch.zeros(4, 6, 9)), (torch.zeros(4, 6, 9), _heads(6, 4, 9)),
                   (_heads(6, 4, 9, pad=3), _heads(6, 4, 9)), (_heads(9, 4, 6).transpose(1, 2), _heads(9, 4, 6, pad=1).transpose(1, 2)),
                   (_heads(9, 4, 6).transpose(1, 2), None), (_heads(6, 8, 9)[::2], _heads(6, 4, 9)), (_heads(6, 4, 1), None), (_heads(1, 4, 9), None)):
        _check(recorder, G, out)
    for sizes, strides in (((4, 6, 9), (8, 36, 1)), ((4, 6, 9), (9, 35, 1)), ((4, 6, 9), (53, 9, 1)), ((2, 6, 9), (1, 36, 1))):  # with elements in common
        with pytest.raises(binding.SageError):
            binding.orthogonalize(torch.zeros(400).as_strided(sizes, strides))
