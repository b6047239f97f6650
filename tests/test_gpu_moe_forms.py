"""The experts of a mixture on the GPU at the sizes, layouts and kernel forms
that prompts and short calls use, against 64 bits."""
import numpy as np
import pytest
import torch

import mx4_reference as ref
import paper_2506_11309_amd as ss
from gpu_helpers import dev
from test_gpu_moe import experts_of, groups_of
from test_gpu_mx4 import check, half, matrix

pytestmark = pytest.mark.gpu


# rows quantised by the product, then by a launch before it
@pytest.mark.parametrize("T,E,k,K,N", [(1, 8, 2, 256, 48), (3, 4, 2, 512, 128), (4, 6, 2, 2048, 1024), (16, 3, 1, 128, 128), (40, 8, 2, 256, 96),
                                       (500, 3, 2, 256, 512)])
def test_swiglu_over_its_own_input(T, E, k, K, N):
    """h in the buffer of x, from its start and from the middle of it."""
    rng = np.random.default_rng(K + T)
    (Wg, k1, wg), (Wu, k2, wu) = matrix(rng, E, N, K), matrix(rng, E, N, K)
    g, (offsets, rows, pos) = groups_of(experts_of(rng, T, E, k, "random"), E)
    x = rng.standard_normal((T, K)).astype(np.float16)
    ws = ss.workspace(ss.moe_mx4_swiglu_workspace_bytes(T, k, E, K, N))
    want = ref.swiglu(x, wg, wu, offsets, rows, k)
    for at in (0, 8 * (T * K // 16)):  # where h begins
        room = torch.zeros(max(T * K, at + T * k * N), dtype=torch.float16, device=dev())
        mine, out = room[:T * K].view(T, K), room[at:at + T * k * N].view(T * k, N)
        mine.copy_(half(x))
        ss.moe_mx4_swiglu(Wg, Wu, mine, g, out, ws)
        check(out, *want)
    assert ss.read_device_error(ws) == 0
