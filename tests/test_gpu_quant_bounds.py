"""Attention over the 8-bit cache at the edges of what its header promises: offsets that make more work than the call has
room for, and how far results may be off."""
import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from quant_helpers import Pool, on_device
from test_gpu_quant_attend import SCALE, _cuda, check, parts_of, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [0x00, 0x3C, 0xFF])
def test_rows_beyond_the_call_are_left_alone(fill):
    """Descending offsets give 101 sequences of 256 tokens where the call has 512 tokens in all.  A hundred of them are the same sequence
    (table, lengths, rows); the last one may have no output, but none that comes out of the workspace."""
    rng = np.random.default_rng(1)
    heads, group, m, n_same, width = 4, 4, 256, 100, 11
    off = np.array([0, m] * n_same + [m, 2 * m], dtype=np.int32)
    batch = len(off) - 1                                     # [0, m), descending, [0, m), ..., [0, m), empty, [m, 2 m)
    lens = np.tile(rng.integers(1000, 1400, (heads, 1)), (1, batch))
    table = np.tile(rng.integers(0, 40, (1, width)).astype(np.int32), (batch, 1))
    pools = [Pool(1, 40, 128, heads) for _ in range(2)]
    for pool in pools:
        pool.codes[:] = rng.integers(0, 127, pool.codes.shape) + 128 * rng.integers(0, 2, pool.codes.shape)
        pool.byte[:] = rng.integers(112, 119, pool.byte.shape)
    q = queries(rng, 2 * m, heads * group, "bf16")
    out, lse = torch.full_like(q, 99.0), torch.full(q.shape[:2], 99.0, device="cuda")
    qs = B.Queries(q, out, _cuda(off), max_q=m, max_len=width * 128, scale=SCALE, lse=lse)
    qc, status = on_device(*pools, table), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(qc, qs) + 256, dtype=torch.uint8, device="cuda").fill_(fill)
    B.skipkv_quant_attend(qc, 0, qs, _cuda(lens.astype(np.int32)), ws, status)
    assert int(status.item()) == B.DEV_BAD_LENGTHS
    check(out[:m], lse[:m], q[:m], [m], lens[:, :1], *pools, table[:1], 128, 0, parts_of("bf16", m, group), heads=[0, 3])
    for h in range(heads):
        mine = out[m:, group * h:group * (h + 1)]
        written = (mine != 99).any(2)
        if bool(written.any()):
            assert bool(written.all())
            check(out[m:], lse[m:], q[m:], [m], lens[:, :1], *pools, table[:1], 128, 0, parts_of("bf16", m, group), heads=[h])
        else:
            assert bool((lse[m:, group * h:group * (h + 1)] == 99).all())
