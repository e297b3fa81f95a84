"""8-bit pools without a GPU: the definition's reference, sizes, refusals (before any GPU work) and launch plans."""
import numpy as np
import pytest

import q8_ref as R
from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W

FMT = pytest.mark.parametrize("fmt", ["e4m3", "int8"])


def _pool(fmt, blocks=64, H=4, D=64, Hkv=None, ptr=0x1000000, nbytes=None):
    cfg = B.make_cfg(blocks, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    return B.KvPool(cfg, ptr, blocks * B.block_bytes(Hkv or H, D, 16, R.FORMATS[fmt]) if nbytes is None else nbytes)


@FMT
def test_reference_rounds_by_at_most_half_a_step(fmt):
    rng = np.random.default_rng(1)
    x = W.f32_to_bf16_bits((rng.standard_normal((400, 64)) * np.exp2(rng.integers(-30, 30, (400, 1)))).astype(np.float32))
    codes, scales = R.quantise(x, fmt)
    f, v = W.bf16_bits_to_f64(x), R.values(codes, scales, fmt)
    e = np.exp2(scales.astype(np.float64) - 127)[:, None]
    a = np.abs(f).max(1, keepdims=True)
    assert (a <= R.TOP[fmt] * e).all() and (a > R.TOP[fmt] * e / 2).all()          # e is the smallest
    half = np.maximum(np.abs(f) * 2.0 ** -4, e * 2.0 ** -10) if fmt == "e4m3" else e / 2
    assert (np.abs(v - f) <= half).all()
    assert np.array_equal(W.bf16_bits_to_f64(W.f32_to_bf16_bits(v.astype(np.float32))), v)  # exact in bf16
    c2, s2 = R.quantise(W.f32_to_bf16_bits(v.astype(np.float32)), fmt)               # quantising a cache's values keeps them
    assert np.array_equal(R.values(c2, s2, fmt), v)


@FMT
@pytest.mark.parametrize("Hkv,D", [(1, 64), (5, 128), (8, 128), (40, 128), (2, 256)])
def test_block_bytes(fmt, Hkv, D):
    p = _pool(fmt, 8, Hkv, D)
    assert p.block_bytes == B.block_bytes(Hkv, D, 16, R.FORMATS[fmt]) == -(-32 * Hkv * (D + 1) // 128) * 128
    with pytest.raises(B.InferceptError) as e:
        _pool(fmt, 8, Hkv, D, nbytes=8 * p.block_bytes - 1)
    assert e.value.code == B.IC_ESIZE
    p.close()


def test_dtypes_that_are_not_built():
    for dtype in (-1, 1, 4, 8, 1 << 20):
        with pytest.raises(B.InferceptError) as e:
            B.KvPool(B.make_cfg(64, 4, 64, dtype=dtype), 0x10000, 1 << 30)
        assert e.value.code == B.IC_EUNSUPPORTED
    for kw in (dict(D=96), dict(D=32)):
        with pytest.raises(B.InferceptError) as e:
            _pool("e4m3", **kw)
        assert e.value.code == B.IC_EUNSUPPORTED


@FMT
def test_read_and_write_refuse_before_any_gpu_work(fmt):
    p = _pool(fmt)
    b = W.make_batch(W.TINY)
    ok = B.HostDesc.from_batch(b)
    k, v = 0x9000000, 0xa000000
    for fn in (p.kv_read_span, p.kv_write_span):
        assert fn(ok, 0, v, check=False) == B.IC_ENULL
        assert fn(ok, k, 0, check=False) == B.IC_ENULL
        assert fn(ok, k + 8, v, check=False) == B.IC_EALIGN
        assert fn(ok, k, v + 2, check=False) == B.IC_EALIGN
        bt = b.block_tables.copy(); bt[2, 0] = 64
        assert fn(B.HostDesc(b.ctx_len, b.q_len, b.q_start, bt, b.scale, b.total_q_rows), k, v, check=False) == B.IC_ERANGE
        bt[2, 0] = -1
        assert fn(B.HostDesc(b.ctx_len, b.q_len, b.q_start, bt, b.scale, b.total_q_rows), k, v, check=False) == B.IC_ERANGE
        assert fn(B.HostDesc(b.ctx_len, b.q_len + 1000, b.q_start, b.block_tables, b.scale, 10 ** 5), k, v, check=False) == B.IC_EINVAL
    rows = b.total_q_rows * 4 * 64 * 2
    assert p.kv_read_span(ok, k, k + rows - 16, check=False) == B.IC_EINVAL              # the two outputs overlap
    assert p.kv_read_span(ok, 0x1000000 + 64 * p.block_bytes - 16, v, check=False) == B.IC_EINVAL   # the pool's own memory
    assert p.kv_read_span(ok, k, 0x1000000 - rows + 16, check=False) == B.IC_EINVAL
    p.close()


@FMT
def test_swap_calls_refuse_before_any_gpu_work(fmt):
    p = _pool(fmt)
    assert p.kv_pack_blocks([64], 0x9000000, 1 << 30, check=False) == B.IC_ERANGE
    assert p.kv_pack_blocks([1, 2], 0x9000000, 2 * p.block_bytes - 1, check=False) == B.IC_ESIZE
    assert p.kv_unpack_blocks([3, 3], 0x9000000, 1 << 30, check=False) == B.IC_EDUP
    assert p.kv_pack_blocks_static([1], 0x1000000, 1 << 30, check=False) == B.IC_EINVAL
    import ctypes as C
    gbps = C.c_double(0)
    ids = np.array([1], dtype=np.int32)
    assert B.lib().ic_paged_read_ceiling(p._h, ids.ctypes.data_as(C.POINTER(C.c_int32)), 1, C.c_void_p(0x9000000), 1, None,
                                         C.byref(gbps)) == B.IC_EUNSUPPORTED             # the probe reads bf16 tiles
    p.close()


def _visits(plan_pool, desc, batch):
    """{(query row): list of key ranges with the number of visits} from the launch plan's row and tile items, and the partial
    slots each row's pieces write."""
    plan = plan_pool.plan_image(desc)
    seen = {r: np.zeros(int(c), dtype=np.int32) for s in range(batch.num_seqs) for r, c in
            ((int(batch.q_start[s]) + i, batch.ctx_len[s] - batch.q_len[s] + i + 1) for i in range(int(batch.q_len[s])))}
    slots = {}
    for seq, qrow, k0, k1, slot, n, pos0, nparts in plan["row_items"]:
        assert 1 <= n and k0 < k1 and k0 % 16 == 0
        for r in range(n):
            lim = pos0 + r + 1
            assert len(seen[qrow + r]) == lim                       # the row's own position
            seen[qrow + r][k0:min(k1, lim)] += 1
            if slot >= 0:
                slots.setdefault(qrow + r, []).append(slot + r * nparts)
    for seq, qrow, n, pos0, k0, k1, slot, nparts in plan["tile_items"]:
        for r in range(n):
            seen[qrow + r][k0:min(k1, pos0 + r + 1)] += 1
            if slot >= 0:
                slots.setdefault(qrow + r, []).append(slot + r * nparts)
    merges = {int(m[0]): list(range(m[1], m[1] + m[2])) for m in plan["merge_items"]}
    return plan, seen, slots, merges


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (6, 2, 128), (16, 2, 128), (32, 1, 128), (24, 1, 64), (64, 8, 128), (4, 2, 256)])
@pytest.mark.parametrize("tuning", [dict(), dict(decode_part_tokens=64, span_part_tokens=128), dict(span_kernel=1), dict(span_kernel=2),
                                    dict(span_kernel=1, decode_part_tokens=64), dict(mfma_min_keys=1)])
def test_plan_covers_every_visible_key_once(fmt, H, Hkv, D, tuning):
    ctx = [1, 5, 16, 17, 100, 1000, 40, 300, 64, 70, 333, 5, 517, 4500]
    q_len = [1, 1, 1, 1, 1, 1, 40, 300, 2, 9, 33, 5, 31, 1]
    blocks = sum(-(-c // 16) for c in ctx) + 3
    batch = W.assemble_batch(H, D, 16, blocks, ctx, q_len, np.random.default_rng(3), num_kv_heads=Hkv)
    p = _pool(fmt, blocks, H, D, Hkv)
    p.set_tuning(**tuning)
    desc = B.HostDesc.from_batch(batch)
    plan, seen, slots, merges = _visits(p, desc, batch)
    for row, n in seen.items():
        assert (n == 1).all(), row
    assert {r: sorted(s) for r, s in slots.items()} == merges       # what is split is merged, every slot written once
    every = sorted(s for m in merges.values() for s in m)
    assert every == list(range(len(every)))
    per_row = max(1, 16 // (H // Hkv))
    assert len(plan["row_items"]) == 0 or plan["row_items"][:, 5].max() <= per_row   # columns of an item: 16
    p.close()


@FMT
def test_short_spans_are_row_items(fmt):
    """Up to three row items of 16 columns (head_dim 256: two); longer ones are tiles, and all of them with span_kernel = 2."""
    for H, Hkv, D, n, tiles in [(4, 4, 128, 48, 0), (4, 4, 128, 49, 1), (64, 8, 128, 6, 0), (64, 8, 128, 7, 1), (32, 1, 64, 3, 0), (32, 1, 64, 4, 1),
                                (4, 4, 256, 32, 0), (4, 4, 256, 33, 1)]:
        blocks = 80
        batch = W.assemble_batch(H, D, 16, blocks, [1000], [n], np.random.default_rng(1), num_kv_heads=Hkv)
        p = _pool(fmt, blocks, H, D, Hkv)
        desc = B.HostDesc.from_batch(batch)
        assert bool(p.plan_query(desc)["tile_items"]) == bool(tiles)
        p.set_tuning(span_kernel=2)
        assert p.plan_query(desc)["tile_items"] > 0
        p.close()


@FMT
def test_plan_of_a_small_workspace(fmt):
    """The splits that only save time are left out where the workspace has no room for them: the unsplit plan's bytes are enough."""
    batch = W.assemble_batch(8, 128, 16, 600, [9000], [1], np.random.default_rng(1))
    p = _pool(fmt, 600, 8, 128)
    desc = B.HostDesc.from_batch(batch)
    assert p.plan_query(desc)["partial_slots"] > 9000 // 4096 + 1
    p.set_tuning(decode_part_tokens=4096)
    assert p.plan_query(desc)["partial_slots"] == 3
    p.close()
