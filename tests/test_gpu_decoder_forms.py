"""Products of 8-bit rows in every form that their sizes choose, with shared sums and without, with a bias and without, in both
types; which forms the sizes reach is checked on the CPU (test_decoder_sizes.py)."""
import pytest
import torch

import paper_2404_02445_amd as P
from tests.test_gpu_decoder import DT, gen, linear_on_gpu, randn, rows8

pytestmark = pytest.mark.gpu

# (tokens, n_out, width).  Up to 16 rows by more than 4096 columns, sums of many stages; the tiles between; sums shared out among blocks
# in each form that shares them, columns off four and widths off every step among them
FORMS = [(1, 28672, 4096), (7, 4099, 1031), (16, 5000, 4111), (9, 4120, 515), (3, 300, 9001), (11, 300, 4097), (16, 4096, 1040), (25, 3000, 2500), (32, 9001, 4100),
         (60, 999, 3000), (64, 6200, 2070), (190, 2900, 5003), (130, 4500, 1500), (100, 14000, 1025), (70, 30001, 200)]
SHARED = [(1, 511, 28672), (8, 1000, 40001), (13, 515, 32769), (16, 33, 131071), (20, 700, 16000), (30, 131, 20001), (64, 513, 14336), (40, 77, 20001), (64, 1024, 12305),
          (100, 301, 9999)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("m,n,k", FORMS + SHARED)
def test_linear_forms(dt, with_bias, m, n, k):
    g = gen(m + n + k)
    x, w = rows8(g, m, k), rows8(g, n, k, extra=16)
    bias = randn(g, n, dt=dt) if with_bias else None
    want, tol = linear_on_gpu(x, w, bias, dt)
    room = torch.empty(m + 2, n + 7, device="cuda", dtype=DT[dt])
    first = None
    for ws in (None, P.alloc_linear8_workspace(x, w, room)):
        for at in (0, 3):                             # (on and off whole vectors)
            room.fill_(7.0)
            out = room[1:m + 1, at:at + n]
            P.mopar_linear8(x, w, out, bias=bias, ws=ws)
            assert bool(((out.double() - want).abs() <= tol).all())
            first = out.clone() if first is None else first
            assert torch.equal(out, first)            # exact sums: the same bits however they are cut
            out.fill_(7.0)
            assert bool((room == 7).all())
