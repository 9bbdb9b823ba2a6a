"""Pins of the row operators' oracle (no GPU): closed forms, finite differences, brute force."""
import itertools

import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from paper_2405_19715_b200 import specdec


def _row(seed, V=13, k=5, rest=True, T=1.3):
    rng = np.random.default_rng(seed)
    t, z = rng.normal(size=V) * 2, rng.normal(size=V) * 2
    y = np.argsort(-t)[:k].astype(np.int32)
    return z, t[y], y, (ro.log_sum_exp(t, T) if rest else None), T, t


def test_top_logits_against_python_sort():
    rng = np.random.default_rng(1)
    z = rng.integers(-3, 4, size=(20, 17)).astype(float)
    z[3, 4] = np.nan
    z[5] = -np.inf
    values, tokens, lse = ro.top_logits(z, 9, 1.0)
    for n in range(20):
        want = sorted(range(17), key=lambda v: (np.isnan(z[n, v]), -np.nan_to_num(z[n, v], neginf=-1e9), v))[:9]
        assert tokens[n].tolist() == want
        ref = torch.logsumexp(torch.tensor(z[n]), 0).item()
        assert (np.isnan(ref) and np.isnan(lse[n])) or ref == lse[n] or abs(ref - lse[n]) < 1e-12


@pytest.mark.parametrize("rest", [True, False])
def test_distill_gradient_against_differences(rest):
    z, v, y, lse, T, _ = _row(3, rest=rest)
    _, g = ro.distill_row(z, v, y, lse, T)
    h = 1e-5
    for i in range(len(z)):
        d = np.zeros_like(z)
        d[i] = h
        num = (ro.distill_row(z + d, v, y, lse, T)[0] - ro.distill_row(z - d, v, y, lse, T)[0]) / (2 * h)
        assert abs(num - g[i]) < 1e-9          # differences are off by h^2 and by 1e-16 / h


def test_distill_of_the_whole_vocabulary_is_the_divergence():
    z, _, _, _, T, t = _row(5)
    p, q = (np.exp(x / T - ro.log_sum_exp(x, T)) for x in (t, z))
    for lse in (None, ro.log_sum_exp(t, T)):
        loss, g = ro.distill_row(z, t, np.arange(len(t)), lse, T)
        assert abs(loss - (p * np.log(p / q)).sum()) < 1e-12
        assert np.allclose(g, (q - p) / T, atol=1e-12)
    assert abs(ro.distill_row(t, t[:4], np.arange(4), ro.log_sum_exp(t, T), T)[0]) < 1e-12      # a draft that agrees


def test_distill_special_rows():
    z, v, y, lse, T, _ = _row(7)
    assert ro.distill_row(z, v, np.full_like(y, -1), lse, T)[0] == 0
    assert np.isnan(ro.distill_row(z, v, np.full_like(y, 2), lse, T)[0])
    assert ro.distill_row(np.full_like(z, -np.inf), v, y, lse, T)[0] == np.inf


def test_beam_select_against_enumeration():
    rng = np.random.default_rng(2)
    B, W, V, M, T = 2, 3, 5, 7, 0.7
    x, s = rng.normal(size=(B, W, V)), rng.normal(size=(B, W)) - 5
    got = ro.beam_select(x, s, M, T)
    for b in range(B):
        every = sorted(((-(s[b, w] + torch.log_softmax(torch.tensor(x[b, w]) / T, 0)[v].item()), w, v) for w, v in itertools.product(range(W), range(V))))[:M]
        assert [e[1:] for e in every] == list(zip(got[1][b].tolist(), got[2][b].tolist()))
        assert np.allclose([-e[0] for e in every], got[0][b], atol=1e-12)
    s[0, 1] = -np.inf
    fin = np.zeros((B, W), np.int32)
    fin[1] = 1
    sc, p, t = ro.beam_select(x, s, W * V, T, fin, 2)
    assert set(t[1, :W].tolist()) == {2} and sorted(p[1, :W].tolist()) == list(range(W))
    # what an ended beam does not end with has no probability, and comes in the order of (beam, token)
    assert list(zip(p[1].tolist(), t[1].tolist()))[W:] == [(w, v) for w in range(W) for v in range(V) if v != 2] and np.all(np.isneginf(sc[1, W:]))
    assert t[0, -V:].tolist() == list(range(V)) and np.all(p[0, -V:] == 1) and np.all(np.isneginf(sc[0, -V:]))


def test_beam_reorder_steps():
    st = np.arange(2 * 3 * 4).reshape(2, 3, 4)
    out = ro.beam_reorder(st, np.array([[2, 0, -1], [9, 1, 0]]), np.array([2, 9]))
    assert out[0].tolist() == [[8, 9, 2, 3], [0, 1, 6, 7], [8, 9, 10, 11]]
    assert out[1].tolist() == [[12, 13, 14, 15], [16, 17, 18, 19], [12, 13, 14, 15]]


# ---- host side of the binding ----------------------------------------------------------------------------------------

def test_state_layouts():
    lay = specdec._state_layout
    c = torch.empty(3, 2, 4, 8, 16, 5, dtype=torch.bfloat16)                     # [L, B, W, H, S, D]
    assert lay(c, 1, 4) == (3, 8, 16, 10, 2 * 4 * 640 * 2, 4 * 640 * 2, 640 * 2, 160)
    assert lay(c, 1, None) == (3, 1, 1, 1280, 10240, 5120, 1280, 0)
    assert lay(c[:, :, :, :, :9], 1, 4)[1:4] == (8, 9, 10)                       # a prefix of the steps
    s = torch.empty(2, 4, 16, 8, 5)                                              # [B, W, S, H, D]
    assert lay(s, 0, 2) == (1, 1, 16, 160, 0, 4 * 640 * 4, 640 * 4, 0)
    assert lay(torch.empty(2, 4, dtype=torch.int32), 0, None) == (1, 1, 1, 4, 0, 16, 4, 0)
    with pytest.raises(ValueError):
        lay(c.transpose(4, 5), 1, 5)                                             # steps whose bytes lie apart
    with pytest.raises(ValueError):
        lay(c, 1, 2)
    with pytest.raises(ValueError):
        lay(c, 5, None)
    with pytest.raises(ValueError):
        lay(torch.empty(4, 4, 2, 3, 8, 8)[::2, :3], 2, None)                     # outer dimensions that do not fold


def test_workspace_size_needs_no_gpu():
    lib = specdec.load_library()
    assert lib.specdec_beam_workspace(1, 4, 32000, 8) == 256 + 256 + 256
    assert lib.specdec_beam_workspace(0, 4, 32000, 8) == 0


def test_null_context_is_an_error():
    lib = specdec.load_library()
    assert lib.specdec_top_logits(None, None, 0, 1, 1, 1, 1, 1.0, None, None, None, None) == specdec.EINVAL
    for f in (lib.specdec_distill, ):
        assert f(None, None, None, None, None) == specdec.EINVAL
    assert lib.specdec_distill_backward(None, None, None, None, None, 1, None) == specdec.EINVAL
    assert lib.specdec_distill_step(None, None, None, None, None, 1, None) == specdec.EINVAL
    assert lib.specdec_beam_reorder(None, None, 1, None, 1, 1, None, None) == specdec.EINVAL
