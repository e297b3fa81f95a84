"""Launch plans of 8-bit pools without a GPU: what the tuning's fields change, and what the pool's size may be."""
import ctypes as C

import numpy as np
import pytest

import q8_ref as R
from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W

FMT = pytest.mark.parametrize("fmt", ["e4m3", "int8"])


def _pool(fmt, blocks, H, D, Hkv=None):
    return B.KvPool(B.make_cfg(blocks, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt]), 0x1000000, blocks * B.block_bytes(Hkv or H, D, 16, R.FORMATS[fmt]))


def _image(pool, desc):
    """The bytes of the descriptor image, and what would be launched."""
    lay, how = B.PlanLayout(), B.PlanLaunchInfo()
    assert B.lib().ic_plan_image(pool._h, C.byref(desc.struct), None, 0, C.byref(lay)) == B.IC_OK
    img = np.zeros(lay.image_bytes, dtype=np.uint8)
    assert B.lib().ic_plan_image(pool._h, C.byref(desc.struct), img.ctypes.data_as(C.c_void_p), img.nbytes, C.byref(lay)) == B.IC_OK
    assert B.lib().ic_plan_launches(pool._h, C.byref(desc.struct), C.byref(how)) == B.IC_OK
    return img.tobytes(), bytes(lay), bytes(how), pool.workspace_bytes(desc)


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(8, 8, 128), (16, 2, 64), (24, 1, 128), (4, 4, 256)])
@pytest.mark.parametrize("tuning", [dict(row_slots=128), dict(row_slots=65536), dict(row_variant=3), dict(row_slots=64, row_variant=1)])
@pytest.mark.parametrize("ctx,q_len", [([3000], [1]), ([3000, 90, 700], [1, 1, 1]), ([2500, 3000, 400], [1, 300, 3])])
def test_fields_of_the_vector_row_kernel_have_no_effect(fmt, H, Hkv, D, tuning, ctx, q_len):
    batch = W.assemble_batch(H, D, 16, 500, ctx, q_len, np.random.default_rng(1), num_kv_heads=Hkv)
    pool, desc = _pool(fmt, 500, H, D, Hkv), B.HostDesc.from_batch(batch)
    plain = _image(pool, desc)
    pool.set_tuning(**tuning)
    assert _image(pool, desc) == plain
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D,ctx,q_len", [(8, 8, 128, [3000, 500], [1, 1]), (16, 2, 64, [3000], [1]), (4, 4, 256, [3000, 500], [1, 1]),
                                               (4, 4, 256, [3000, 400], [1, 300])])
def test_asking_for_a_pair_that_there_is_none_of_changes_nothing(fmt, H, Hkv, D, ctx, q_len):
    """row_launch = 2: no tiles to run beside, or head_dim 256."""
    batch = W.assemble_batch(H, D, 16, 500, ctx, q_len, np.random.default_rng(1), num_kv_heads=Hkv)
    pool, desc = _pool(fmt, 500, H, D, Hkv), B.HostDesc.from_batch(batch)
    plain = _image(pool, desc)
    for row_launch in (1, 2) + ((3,) if D == 256 else ()):
        pool.set_tuning(row_launch=row_launch)
        assert _image(pool, desc) == plain
    pool.close()


@FMT
def test_cache_slots_fit_32_bits(fmt):
    """Slots are block * 16 + slot in an int32: the last one of 2^27 blocks is 2^31 - 1; a block more would be written nowhere."""
    H, D, most = 1, 64, 1 << 27
    bb = B.block_bytes(H, D, 16, R.FORMATS[fmt])
    p = B.KvPool(B.make_cfg(most, H, D, dtype=R.FORMATS[fmt]), 0x1000000, most * bb)
    desc = B.HostDesc([16], [16], [0], np.array([[most - 1]], np.int32), 1.0, 16)
    dst = p.plan_image(desc)["row_dst"]
    assert dst[0] == (most - 1) * 16 and dst[15] == 2 ** 31 - 1
    p.close()
    with pytest.raises(B.InferceptError) as e:
        B.KvPool(B.make_cfg(most + 1, H, D, dtype=R.FORMATS[fmt]), 0x1000000, (most + 1) * bb)
    assert e.value.code == B.IC_EINVAL
    cfg = B.make_cfg(most + 1, H, D, dtype=R.FORMATS[fmt])
    assert B.lib().ic_check_batch(C.byref(cfg), C.byref(desc.struct)) == B.IC_EINVAL


@FMT
@pytest.mark.parametrize("H,Hkv", [(32, 32), (64, 16)])
def test_whole_rows_once_every_place_has_two_items(fmt, H, Hkv):
    """One long row among short ones stays whole from two items a place on: 2 x 2 x 256 workgroups, at head_dim 64, where a CU has four, twice that."""
    for D, items in ((64, 2048), (128, 1024), (256, 1024)):
        for n in (items // Hkv - 1, items // Hkv):
            ctx = [4000] + [300] * (n - 1)
            batch = W.assemble_batch(H, D, 16, sum(-(-c // 16) for c in ctx) + 5, ctx, [1] * n, np.random.default_rng(1), num_kv_heads=Hkv)
            pool = _pool(fmt, batch.pool_blocks, H, D, Hkv)
            assert (pool.plan_image(B.HostDesc.from_batch(batch))["row_part_tokens"] < 4000) == (n * Hkv < items)
            pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D,ctx,q_len", [(8, 8, 128, [3500, 100], [1, 1]), (16, 2, 64, [4000], [1]), (4, 4, 256, [3000, 900], [1, 300])])
def test_a_workspace_without_room_for_the_splits_is_enough(fmt, H, Hkv, D, ctx, q_len):
    """A call that gets the bytes of the unsplit plan is planned without the splits; with fewer it is refused.  (No GPU: a call that is not refused
    fails where it asks for pinned memory.)"""
    import torch
    if torch.cuda.device_count() > 0:
        pytest.skip("the call would run on made-up addresses")
    batch = W.assemble_batch(H, D, 16, 600, ctx, q_len, np.random.default_rng(1), num_kv_heads=Hkv)
    pool, desc = _pool(fmt, 600, H, D, Hkv), B.HostDesc.from_batch(batch)
    full = pool.workspace_bytes(desc)
    pool.set_tuning(decode_part_tokens=4096, span_part_tokens=1 << 20)
    least = pool.workspace_bytes(desc)
    assert pool.plan_query(desc)["partial_slots"] == 0
    pool.set_tuning()
    assert pool.plan_query(desc)["partial_slots"] > 0 and least < full
    at = [0x9000000, 0xa000000, 0xb000000]
    assert pool.paged_attn_mixed(desc, *at, least, check=False) not in (B.IC_OK, B.IC_ESIZE)
    assert pool.paged_attn_mixed(desc, *at, least - 256, check=False) == B.IC_ESIZE
    pool.close()


@pytest.mark.parametrize("dtype", [B.IC_DTYPE_BF16, B.IC_DTYPE_E4M3, B.IC_DTYPE_INT8])
@pytest.mark.parametrize("ctx", [17, 2 ** 31 - 16, 2 ** 31 - 15, 2 ** 31 - 1])
def test_a_context_longer_than_its_table(dtype, ctx):
    """Up to the largest int32, where rounding up to blocks would overflow."""
    cfg = B.make_cfg(64, 4, 64, dtype=dtype)
    desc = B.HostDesc([ctx], [1], [0], np.zeros((1, 1), np.int32), 1.0, 1)
    assert B.lib().ic_check_batch(C.byref(cfg), C.byref(desc.struct)) == B.IC_ESIZE
