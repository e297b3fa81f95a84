"""Batches with more work items than a launch may have threads for are refused before anything is launched.  Without a GPU: the device
addresses are made up, and a call that is not refused ends where it asks for memory."""
import numpy as np
import pytest
import torch

from paper_2402_01869_amd import binding as B

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="calls that are not refused would run on made-up addresses")
PTR = 0x7000_0000_0000


def _call(H, Hkv, D, rows, ctx=1, tuning=None):
    pool = B.KvPool(B.make_cfg(64, H, D, num_kv_heads=Hkv), PTR, 64 * B.block_bytes(Hkv, D))
    if tuning:
        pool.set_tuning(**tuning)
    n_blocks = -(-ctx // 16)
    desc = B.HostDesc(np.full(rows, ctx, np.int32), np.ones(rows, np.int32), np.arange(rows, dtype=np.int32), np.zeros((rows, n_blocks), np.int32), 1.0, rows,
                      flags=B.IC_FLAG_TRUSTED)
    how = pool.plan_launches(desc)
    rc = pool.paged_attn_mixed(desc, PTR + (1 << 30), PTR + (2 << 30), PTR + (3 << 30), 1 << 40, check=False)
    with pytest.raises(B.InferceptError) as e:
        pool.plan_create(desc, PTR + (3 << 30), 1 << 40)
    assert e.value.code == rc
    pool.close()
    return how, rc


@pytest.mark.parametrize("H,Hkv,ctx", [(40, 40, 1), (256, 256, 30), (64, 64, 16)])
def test_one_workgroup_per_short_row(H, Hkv, ctx):
    most = (1 << 32) // 256 // H                                 # 2^32 threads: one too many
    most -= most * H * 256 == 1 << 32
    how, rc = _call(H, Hkv, 64, most + 1, ctx)
    assert how["row_launch"] == 1 and rc == B.IC_EINVAL
    how, rc = _call(H, Hkv, 64, most, ctx)
    assert rc != B.IC_EINVAL                                     # (whatever a machine without the memory says)


def test_persistent_rows_have_no_such_limit():
    how, rc = _call(256, 256, 64, 66000, 30, dict(row_launch=2))
    assert how["row_launch"] == 2 and rc != B.IC_EINVAL


def test_one_workgroup_per_row_of_a_group():
    how, rc = _call(512, 256, 64, 65536, 64)
    assert how["group_launch"] == 1 and rc == B.IC_EINVAL
    how, rc = _call(512, 256, 64, 65535, 64)
    assert rc != B.IC_EINVAL
