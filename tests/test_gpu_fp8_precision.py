"""The mean square of the 8-bit products' errors on the GPU, in every form of their
plan: sums, experts' rows and shares of K kept in fewer than 32 bits, or scales in fewer
than theirs, exceed it."""
import numpy as np
import pytest
import torch

import fp8_precision as prec
import paper_2506_11309_amd as ss
import test_gpu_fp8_forms as forms
from gpu_helpers import dev, up
from test_gpu_fp8_forms import Matrix
from test_gpu_moe import experts_of, groups_of
from test_gpu_moe_forms import expert_edges, sample
from test_gpu_mx4 import half

pytestmark = pytest.mark.gpu


def operands(m):
    """The sampled columns of a matrix, or of each expert's."""
    c, s = m.keep[0].index_select(-2, m.gpu_at).cpu().numpy(), m.keep[1].cpu().numpy()
    each = [prec.Operand(c[e], s[e][m.at // 128]) for e in range(len(c))] if c.ndim == 3 else [prec.Operand(c, s[m.at // 128])]
    return each


def picked(t, rows, m):
    return t[torch.from_numpy(rows).to(dev())][:, m.gpu_at]


@pytest.mark.parametrize("M,K,N,form,split", forms.GEMM)
@pytest.mark.parametrize("residual", [False, True])
def test_gemm(M, K, N, form, split, residual):
    rng = np.random.default_rng(M + K + 1)
    m = Matrix(M + 7, 1, N, K, one=True)
    x = rng.standard_normal((M, K)).astype(np.float16)
    r = rng.standard_normal((M, N)).astype(np.float16) * 4 if residual else None
    y = torch.empty(M, N, dtype=torch.float16, device=dev())
    ss.fp8_gemm(m.W, half(x), y, ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N)), residual=half(r) if residual else None)
    rows = sample(M, count=60)
    prec.close(picked(y, rows, m), *prec.gemm(x[rows], operands(m)[0], r[np.ix_(rows, m.at)] if residual else None))


@pytest.mark.parametrize("T,E,k,K,N,kind,form", forms.SWIGLU)
def test_swiglu(T, E, k, K, N, kind, form):
    rng = np.random.default_rng(T + E + K + 2)
    g, u = Matrix(T + 7, E, N, K), Matrix(T + 8, E, N, K)
    u.at, u.gpu_at = g.at, g.gpu_at
    groups, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    h = torch.empty(T * k, N, dtype=torch.float16, device=dev())
    ss.moe_fp8_swiglu(g.W, u.W, half(x), groups, h, ss.workspace(ss.moe_fp8_swiglu_workspace_bytes(T, k, E, K, N)))
    places = sample(offsets[-1], expert_edges(offsets) if E < 20 else (), 60)
    prec.close(picked(h, places, g), *prec.swiglu(x, operands(g), operands(u), offsets, rows, k, places))


@pytest.mark.parametrize("T,E,k,K,N,kind,form,split", forms.DOWN)
@pytest.mark.parametrize("residual", [False, True])
def test_down(T, E, k, K, N, kind, form, split, residual):
    rng = np.random.default_rng(T + E + K + 3)
    m = Matrix(T + 7, E, N, K)
    groups, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, kind), E)
    h = rng.standard_normal((T * k, K)).astype(np.float16)
    p = rng.random((T, k)).astype(np.float32)
    r = rng.standard_normal((T, N)).astype(np.float16) if residual else None
    y = torch.empty(T, N, dtype=torch.float16, device=dev())
    ss.moe_fp8_down(m.W, half(h), groups, up(p), y, ss.workspace(ss.moe_fp8_down_workspace_bytes(T, k, E, K, N)), residual=half(r) if residual else None)
    tokens = sample(T, count=40)
    prec.close(picked(y, tokens, m), *prec.down(h, operands(m), offsets, pos, p, r[:, m.at] if residual else None, tokens))


def test_gemm_of_a_deep_matrix():
    """The most columns of the tests: 385 groups of 128."""
    K, N = forms.LARGE_K, 2064
    m = Matrix(5, 1, N, K, one=True)
    rng = np.random.default_rng(13)
    for M in (5, 40, 400):
        x = rng.standard_normal((M, K)).astype(np.float16)
        y = torch.empty(M, N, dtype=torch.float16, device=dev())
        ss.fp8_gemm(m.W, half(x), y, ss.workspace(ss.fp8_gemm_workspace_bytes(M, K, N)))
        rows = sample(M, count=40)
        prec.close(picked(y, rows, m), *prec.gemm(x[rows], operands(m)[0]))
