"""Decode over shared prefixes of many columns (those that go through shared memory) against the plain 64-bit attention, with inputs in which
what could go wrong decides results: weights that cancel, and keys at the borders that each carry a column's result.

Tolerances: a rounding to a type is off by half a step (finfo.eps / 2 of the value); weights are held in 16 bits and more, cut
off below 2^-15 of themselves; sums and scores as in tests/kv_model.py."""
import torch
import pytest

import paper_2502_11880_amd as B
from tests import kv_model as M
from tests.test_gpu_attn_shared import DEV, Groups

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0 ** -15


def _half_step(io):
    return torch.finfo(M.DTYPES[io]).eps / 2


@pytest.mark.parametrize("D,page,dtype", [(128, 64, "bf16"), (100, 16, "f16"), (64, 32, "bf16"), (48, 128, "f16"), (256, 64, "bf16"), (132, 32, "f16")])
def test_weights_keep_their_bits(D, page, dtype):
    """Two neighbouring keys of nearly equal weight and opposite values: what is left is small, and an error of a weight shows in it
    whole.  All other keys have weights below e^-40, 16000 of them together below 2^-43: they are not in the sums."""
    print("case: wide weights", D, page, dtype, flush=True)
    prefix, members, H = 16000, 9, 256
    g = Groups([(members, prefix)], [prefix + 3 * s for s in range(members)], 1, D, page, dtype, seed=D)
    b = g.b
    first, second = 4000, 4010
    gen = torch.Generator().manual_seed(D)
    value = torch.randn(D, generator=gen).to(b.dtype)
    for k in b.k:
        k.zero_()
        k[:, 0, 0] = -40.0
    b.k[0][first, 0, 0] = b.k[0][second, 0, 0] = 0.0
    b.k[0][second, 0, 1] = -1.0
    b.v[0][first, 0], b.v[0][second, 0] = value, -value
    g.write()
    q = torch.zeros(members, H, D)
    q[:, :, 0] = 1.0
    q[:, :, 1] = 0.005 + 0.06 * torch.rand(members, H, generator=gen)
    q = q.to(b.dtype)
    out = g.run(H, q.view(members, H * D).to(DEV), 1.0).cpu().view(members, H, D)
    want, tol = M.attention(q, b.k[0][[first, second]], b.v[0][[first, second]], torch.ones(members, 2, dtype=torch.bool), 1.0, _half_step(dtype), WEIGHTS)
    M.check(out, want, tol, "two keys")
