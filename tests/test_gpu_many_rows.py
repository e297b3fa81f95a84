"""Calls on more query rows than one launch has threads for: a launch takes fewer than 2^32, 16 bytes each."""
import numpy as np
import pytest
import torch

from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W
from gpu_common import DEV, from_dev_bits

pytestmark = pytest.mark.gpu


def test_append_and_read_back_on_64_gib_of_rows():
    """2^22 rows of 8 KiB of keys and as much of values, of which sequences own a few at the start, around the first launch's end and at the end."""
    H, D, total = 16, 256, (1 << 22) + 100
    starts, n = [0, (1 << 22) - 40, (1 << 22) + 60], 40
    rng = np.random.default_rng(1)
    batch = W.assemble_batch(H, D, 16, 20, [n] * 3, [n] * 3, rng)
    desc = B.HostDesc(batch.ctx_len, batch.q_len, starts, batch.block_tables, batch.scale, total)
    t = torch.zeros((20, 2, H, 16, D), dtype=torch.int16, device=DEV)
    pool = B.KvPool.from_tensor(t, H, D)
    k, v = (torch.empty((total, H, D), dtype=torch.int16, device=DEV) for _ in range(2))
    new = rng.integers(-2 ** 15, 2 ** 15, (2, 3, n, H, D)).astype(np.int16)
    for i, rows in enumerate((k, v)):
        for s, r0 in enumerate(starts):
            rows[r0:r0 + n] = torch.from_numpy(new[i, s]).to(DEV)
    torch.cuda.synchronize()
    pool.kv_write_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    host = from_dev_bits(t).view(np.int16)
    for s in range(3):
        for tok in range(n):
            b = batch.block_tables[s, tok // 16]
            for i in range(2):
                assert np.array_equal(host[b, i, :, tok % 16], new[i, s, tok])
    for rows in (k, v):
        for r0 in starts:
            rows[r0:r0 + n].zero_()
    torch.cuda.synchronize()
    pool.kv_read_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    for i, rows in enumerate((k, v)):
        for s, r0 in enumerate(starts):
            assert np.array_equal(from_dev_bits(rows[r0:r0 + n]).view(np.int16), new[i, s])
    pool.close()
    del k, v
    torch.cuda.empty_cache()


def test_pack_and_unpack_of_64_gib():
    """A list of more blocks than one launch moves, out of a pool and back into it in another order."""
    H, D, blocks = 40, 128, 210000
    bb = B.block_bytes(H, D)
    t = torch.empty((blocks, bb // 8), dtype=torch.int64, device=DEV)
    t[:, 0] = torch.arange(blocks, device=DEV)                   # every block has its number at both ends
    t[:, -1] = -torch.arange(blocks, device=DEV) - 1
    pool = B.KvPool.from_tensor(t, H, D)
    rng = np.random.default_rng(2)
    ids = rng.permutation(blocks).astype(np.int32)
    staging = torch.zeros((blocks, bb // 8), dtype=torch.int64, device=DEV)
    torch.cuda.synchronize()
    pool.kv_pack_blocks(ids, staging.data_ptr(), blocks * bb)
    torch.cuda.synchronize()
    assert np.array_equal(staging[:, 0].cpu().numpy(), ids) and np.array_equal(staging[:, -1].cpu().numpy(), -ids.astype(np.int64) - 1)
    to = rng.permutation(blocks).astype(np.int32)
    pool.kv_unpack_blocks(to, staging.data_ptr(), blocks * bb)
    torch.cuda.synchronize()
    want = np.empty(blocks, dtype=np.int64)
    want[to] = ids
    assert np.array_equal(t[:, 0].cpu().numpy(), want) and np.array_equal(t[:, -1].cpu().numpy(), -want - 1)
    pool.close()
    del t, staging
    torch.cuda.empty_cache()
