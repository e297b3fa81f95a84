"""8-bit pools on the GPU: kv_write_span and kv_read_span bit for bit, attention against 64 bits, and their use together.

Tolerances of attention.  A bf16 result is off by at most half a step, 2^-8 of its value.  An error of the weights, relative d, moves the
result by at most 2 d times the mean distance of the values from it (dev).  Row kernel: weights keep 16 bits of significand (2^-17), their
exponents are fp32 (products of 128 numbers of magnitude about 1 and outliers of 4 summed in fp32: under 2e-4, mostly 1e-6): 2 d <= 1e-3.
Tile kernel: weights are rounded to bf16 and the sum counts them as rounded: 2^-8 dev, plus the same 1e-3."""
import numpy as np
import pytest
import torch

import q8_ref as R
from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W
from gpu_common import DEV, from_dev_bits, to_dev_bits

pytestmark = pytest.mark.gpu
FMT = pytest.mark.parametrize("fmt", ["e4m3", "int8"])


def _pool(pool_bytes, H, Hkv, D, fmt):
    t = torch.from_numpy(pool_bytes).to(DEV)
    return B.KvPool.from_tensor(t, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt]), t


def _run(pool, batch, q_bits, ws_bytes=None, stream=0, flags=0):
    desc = B.HostDesc.from_batch(batch, flags=flags)
    q = to_dev_bits(q_bits)
    out = torch.full(q_bits.shape, 0x7FFF, dtype=torch.int16, device=DEV)
    need = pool.workspace_bytes(desc) if ws_bytes is None else ws_bytes
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.paged_attn_mixed(desc, q.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    torch.cuda.synchronize()
    return from_dev_bits(out)


def _close(got_bits, want, dev, weights=2.0 ** -8):
    got = W.bf16_bits_to_f64(got_bits)
    assert np.isfinite(got).all()
    bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (weights + 1e-3) * dev + 1e-6
    worst = np.max(np.abs(got - want) / bound)
    assert worst <= 1.0, worst


ROWS_ONLY = 0.0  # weights of the row kernel: nothing beyond the 1e-3


# ------------------------------------------------------------------------------------------ writing and reading back
@FMT
@pytest.mark.parametrize("H,D", [(1, 64), (5, 64), (3, 128), (2, 256)])
def test_write_is_the_definition(fmt, H, D):
    ctx, q_len = [1, 15, 16, 17, 33, 64, 100, 40, 129], [1, 1, 1, 1, 1, 1, 1, 40, 33]
    rng = np.random.default_rng(H + D)
    batch = W.assemble_batch(H, D, 16, 40, ctx, q_len, rng)
    rows = batch.total_q_rows + 3                                # trailing rows no sequence owns
    x = rng.standard_normal((2, rows, H, D)) * np.exp2(rng.integers(-40, 40, (2, rows, H, 1)).astype(np.float64))
    top = R.TOP[fmt]
    x[0, 0] = 0.0                                                # edges: zeros, the range's ends, ties, tiny, huge, not finite
    x[0, 1, 0] = top
    x[0, 2, 0] = np.where(np.arange(D) % 2, -top, top / 2)
    x[0, 3, 0, :] = np.arange(D) / 2.0
    x[0, 4, 0] = 1e-38
    x[0, 5, 0] = 2.0 ** -130
    x[0, 6, 0, 0] = 3.0e38
    x[1, 0, 0, D - 1] = np.nan
    x[1, 1, 0, 0] = np.inf
    x[1, 2, 0, D // 2] = -np.inf
    x[1, 3, 0] = np.arange(D) - D / 2 + 0.5
    new = W.f32_to_bf16_bits(x.astype(np.float32))
    start = rng.integers(0, 256, (40, B.block_bytes(H, D, 16, R.FORMATS[fmt])), dtype=np.uint8)
    want = start.copy()
    R.write(want, batch, new[0], new[1], fmt)
    pool, t = _pool(start.copy(), H, H, D, fmt)
    desc = B.HostDesc(batch.ctx_len, batch.q_len, batch.q_start, batch.block_tables, batch.scale, rows)
    k, v = to_dev_bits(new[0]), to_dev_bits(new[1])
    pool.kv_write_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    got = t.cpu().numpy()
    gc, gs = R.split(got, H, D)
    wc, ws = R.split(want, H, D)
    assert np.array_equal(gs, ws)
    # -0 rounds to a code of its own in e4m3; the value is what counts
    assert np.array_equal(R.code_values(fmt)[gc], R.code_values(fmt)[wc], equal_nan=True)
    untouched = np.ones(got.shape, dtype=bool)
    for view, width in zip(R.split(untouched, H, D), (4, 3)):
        for s in range(batch.num_seqs):
            for tok in range(int(batch.ctx_len[s] - batch.q_len[s]), int(batch.ctx_len[s])):
                b, slot = batch.block_tables[s, tok // 16], tok % 16
                view[b, :, :, slot] = False
    assert np.array_equal(got[untouched], start[untouched])
    pool.close()


@FMT
@pytest.mark.parametrize("H,D", [(1, 64), (3, 128), (2, 256)])
def test_read_gives_every_code_its_value(fmt, H, D):
    rng = np.random.default_rng(D)
    batch = W.assemble_batch(H, D, 16, 60, [1, 16, 17, 250, 300, 31], [1, 16, 5, 250, 1, 31], rng)
    pool_bytes = rng.integers(0, 256, (60, B.block_bytes(H, D, 16, R.FORMATS[fmt])), dtype=np.uint8)
    _, scales = R.split(pool_bytes, H, D)
    scales[...] = rng.choice(np.r_[27:250, 255], scales.shape)
    pool, t = _pool(pool_bytes, H, H, D, fmt)
    rows = batch.total_q_rows + 2
    desc = B.HostDesc(batch.ctx_len, batch.q_len, batch.q_start, batch.block_tables, batch.scale, rows)
    k, v = (torch.full((rows, H, D), 0x1234, dtype=torch.int16, device=DEV) for _ in range(2))
    pool.kv_read_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    for i, out in enumerate((k, v)):
        got = from_dev_bits(out)
        assert (got[-2:] == 0x1234).all()
        for s in range(batch.num_seqs):
            n, r0 = int(batch.q_len[s]), int(batch.q_start[s])
            want = R.context(pool_bytes, batch, s, H, D, fmt)[i][-n:]
            with np.errstate(over="ignore"):
                want = want.astype(np.float32).astype(np.float64)      # a value may overflow: 2^122 times a large code
            assert np.array_equal(W.bf16_bits_to_f64(got[r0:r0 + n]), want, equal_nan=True)
    pool.close()


@pytest.mark.parametrize("H,D", [(3, 64), (5, 128), (2, 256)])
def test_read_of_a_bf16_pool_is_the_append_the_other_way_round(H, D):
    rng = np.random.default_rng(9)
    batch = W.assemble_batch(H, D, 16, 60, [5, 16, 33, 200], [1, 16, 33, 77], rng)
    bits = rng.integers(0, 1 << 16, W.pool_shape(60, H, 16, D), dtype=np.uint16)
    t = to_dev_bits(bits)
    pool = B.KvPool.from_tensor(t, H, D)
    desc = B.HostDesc.from_batch(batch)
    k, v = (torch.zeros((batch.total_q_rows, H, D), dtype=torch.int16, device=DEV) for _ in range(2))
    pool.kv_read_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    for s in range(batch.num_seqs):
        for i in range(int(batch.q_len[s])):
            tok, row = int(batch.ctx_len[s] - batch.q_len[s]) + i, int(batch.q_start[s]) + i
            b = batch.block_tables[s, tok // 16]
            assert np.array_equal(from_dev_bits(k)[row], bits[b, 0, :, tok % 16])
            assert np.array_equal(from_dev_bits(v)[row], bits[b, 1, :, tok % 16])
    # a read's list is not a write's check: two sequences on one slot may be read, never written
    bt = batch.block_tables.copy(); bt[1] = bt[0]
    dup = B.HostDesc([16, 16], [16, 16], [0, 16], bt[:2], batch.scale, batch.total_q_rows)
    assert pool.kv_read_span(dup, k.data_ptr(), v.data_ptr()) == B.IC_OK
    assert pool.kv_write_span(dup, k.data_ptr(), v.data_ptr(), check=False) == B.IC_EDUP
    torch.cuda.synchronize()
    pool.close()


@FMT
def test_a_context_moves_between_pools_without_loss(fmt):
    """8-bit cache -> bf16 rows -> bf16 cache and another 8-bit cache: the same values."""
    H, D = 4, 128
    rng = np.random.default_rng(4)
    batch = W.assemble_batch(H, D, 16, 40, [200, 16, 90], [200, 16, 90], rng)
    desc = B.HostDesc.from_batch(batch)
    a, ta = _pool(R.random_pool(batch, H, D, fmt, rng), H, H, D, fmt)
    b, tb = _pool(R.empty_pool(40, H, D), H, H, D, fmt)
    c = B.KvPool.from_tensor(torch.zeros((40, 2, H, 16, D), dtype=torch.int16, device=DEV), H, D)
    rows = [[torch.zeros((batch.total_q_rows, H, D), dtype=torch.int16, device=DEV) for _ in range(2)] for _ in range(3)]
    a.kv_read_span(desc, rows[0][0].data_ptr(), rows[0][1].data_ptr())
    for pool, out in ((b, rows[1]), (c, rows[2])):
        pool.kv_write_span(desc, rows[0][0].data_ptr(), rows[0][1].data_ptr())
        pool.kv_read_span(desc, out[0].data_ptr(), out[1].data_ptr())
    torch.cuda.synchronize()
    for i in range(2):
        first = W.bf16_bits_to_f64(from_dev_bits(rows[0][i]))
        for out in rows[1:]:
            assert np.array_equal(first, W.bf16_bits_to_f64(from_dev_bits(out[i])))
    for p in (a, b, c):
        p.close()


# ------------------------------------------------------------------------------------------ attention
@FMT
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (3, 3, 128), (2, 2, 256), (6, 2, 128), (16, 2, 64), (16, 2, 128), (4, 2, 256), (24, 1, 128), (32, 1, 64),
                                     (40, 2, 128)])
@pytest.mark.parametrize("part", [0, 64])
def test_decode_rows(fmt, H, Hkv, D, part):
    ctx = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 129, 257, 1000]
    rng = np.random.default_rng(H * D + Hkv)
    blocks = sum(-(-c // 16) for c in ctx) + 5
    batch = W.assemble_batch(H, D, 16, blocks, ctx, [1] * len(ctx), rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((len(ctx), H, D), rng)
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    pool.set_tuning(decode_part_tokens=part)
    got = _run(pool, batch, q)
    _close(got, *R.attention(pool_bytes, batch, q, Hkv, fmt), weights=ROWS_ONLY)
    assert np.array_equal(got, _run(pool, batch, q))             # the same bits again
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 64), (3, 3, 128), (2, 2, 256), (6, 2, 128), (16, 2, 128), (8, 1, 256), (32, 1, 128)])
@pytest.mark.parametrize("tuning", [dict(), dict(span_part_tokens=64, decode_part_tokens=64), dict(span_kernel=1), dict(span_kernel=2), dict(mfma_min_keys=1),
                                    dict(row_launch=3), dict(row_launch=2, decode_part_tokens=64, span_part_tokens=64), dict(serial_spans=1)])
def test_chunks_and_decode_rows(fmt, H, Hkv, D, tuning):
    ctx = [70, 2, 40, 300, 64, 200, 333, 130, 5, 90]
    q_len = [1, 2, 40, 130, 33, 3, 70, 17, 1, 31]
    rng = np.random.default_rng(H * D + Hkv + 1)
    blocks = sum(-(-c // 16) for c in ctx) + 5
    batch = W.assemble_batch(H, D, 16, blocks, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    pool.set_tuning(**tuning)
    got = _run(pool, batch, q)
    _close(got, *R.attention(pool_bytes, batch, q, Hkv, fmt), weights=ROWS_ONLY if tuning.get("span_kernel") == 1 else 2.0 ** -8)
    assert np.array_equal(got, _run(pool, batch, q))
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D,n", [(8, 8, 128, 40), (8, 8, 64, 40), (16, 2, 128, 60)])
def test_rows_and_tiles_side_by_side(fmt, H, Hkv, D, n):
    """The pair of kernels as a plan of its own choice, again and again from one plan: more work items than places."""
    rng = np.random.default_rng(17)
    ctx = list(rng.integers(100, 900, n)) + [400, 600, 300]
    q_len = [1] * n + [300, 520, 100]
    blocks = sum(-(-int(c) // 16) for c in ctx) + 5
    batch = W.assemble_batch(H, D, 16, blocks, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    want = R.attention(pool_bytes, batch, q, Hkv, fmt)
    pool.set_tuning(serial_spans=1)
    alone = _run(pool, batch, q)
    _close(alone, *want)
    pool.set_tuning(row_launch=2)
    desc = B.HostDesc.from_batch(batch)
    assert pool.plan_image(desc)["side_by_side"] == 1
    qt, ws = to_dev_bits(q), torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = pool.plan_create(desc, ws.data_ptr(), ws.numel(), st.cuda_stream)
    outs = [torch.zeros((len(q), H, D), dtype=torch.int16, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    for out in outs:
        pool.paged_attn_planned(plan, qt.data_ptr(), out.data_ptr(), st.cuda_stream)
    st.synchronize()
    for out in outs:
        assert torch.equal(out, outs[0])
    _close(from_dev_bits(outs[0]), *want)
    plan.close()
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (2, 2, 128), (1, 1, 256), (8, 1, 128)])
def test_chunk_longer_than_a_tile(fmt, H, Hkv, D):
    ctx, q_len = [700, 600], [600, 300]
    rng = np.random.default_rng(5)
    batch = W.assemble_batch(H, D, 16, 90, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    want = R.attention(pool_bytes, batch, q, Hkv, fmt)
    for part in (0, 256, 1 << 20):
        pool.set_tuning(span_part_tokens=part)
        _close(_run(pool, batch, q), *want)
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (2, 2, 128), (1, 1, 256), (8, 2, 128)])
@pytest.mark.parametrize("which", [0, 1])
def test_nan_vectors_show_in_the_rows_that_see_them(fmt, H, Hkv, D, which):
    """which: a key or a value that is not finite, at positions inside a chunk and before a decode row."""
    ctx, q_len, at = [300, 200, 70, 90], [200, 1, 20, 64], [211, 37, 61, 40]
    rng = np.random.default_rng(6)
    batch = W.assemble_batch(H, D, 16, 60, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    codes, scales = R.split(pool_bytes, Hkv, D)
    want, dev = R.attention(pool_bytes, batch, q := W.randn_bf16((sum(q_len), H, D), rng), Hkv, fmt)
    for s, t in enumerate(at):
        b = batch.block_tables[s, t // 16]
        codes[b, which, 0, t % 16] = 0                           # K/V head 0 only
        scales[b, 0, which, t % 16] = 255
        first = max(0, t - (ctx[s] - q_len[s]))                  # the first row that sees it
        want[batch.q_start[s] + first:batch.q_start[s] + q_len[s], :H // Hkv] = np.nan
    for tuning in (dict(), dict(span_kernel=1), dict(span_part_tokens=64, decode_part_tokens=64)):
        pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
        pool.set_tuning(**tuning)
        got = W.bf16_bits_to_f64(_run(pool, batch, q))
        hit = np.isnan(want)
        assert np.isnan(got[hit]).all()
        bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -8 + 1e-3) * dev + 1e-6
        assert (np.abs(got - want)[~hit] <= bound[~hit]).all()
        pool.close()


@FMT
def test_large_and_small_scores(fmt):
    """Scores hundreds apart, one key that takes all the weight, and keys of zeros: the running maximum moves and the sums with it."""
    H, D, ctx = 2, 128, [500, 400, 300]
    rng = np.random.default_rng(8)
    batch = W.assemble_batch(H, D, 16, 80, ctx, [1, 200, 10], rng)
    pool_bytes = R.random_pool(batch, H, D, fmt, rng)
    _, scales = R.split(pool_bytes, H, D)
    for s in range(3):
        for t in range(0, ctx[s], 37):
            scales[batch.block_tables[s, t // 16], :, 0, t % 16] += np.uint8(t // 37 % 5)
    codes, _ = R.split(pool_bytes, H, D)
    codes[batch.block_tables[1, 2], 0] = 0
    q = W.randn_bf16((211, H, D), rng)
    pool, _ = _pool(pool_bytes, H, H, D, fmt)
    # scores up to a few hundred: the fp32 exponent is then good to 2^-24 of their size, 2e-5 a product's rounding of it
    _close(_run(pool, batch, q), *R.attention(pool_bytes, batch, q, H, fmt))
    pool.close()


@FMT
def test_query_rows_nobody_owns_and_shared_blocks(fmt):
    H, D = 4, 128
    rng = np.random.default_rng(12)
    batch = W.assemble_batch(H, D, 16, 60, [200, 200, 90], [1, 60, 40], rng)
    batch.block_tables[1] = batch.block_tables[0]                # two sequences on the same blocks
    batch.q_start[:] = [100, 7, 200]
    pool_bytes = R.random_pool(batch, H, D, fmt, rng)
    q = W.randn_bf16((260, H, D), rng)
    want, dev = R.attention(pool_bytes, batch, q, H, fmt)
    pool, _ = _pool(pool_bytes, H, H, D, fmt)
    desc = B.HostDesc(batch.ctx_len, batch.q_len, batch.q_start, batch.block_tables, batch.scale, 260)
    out = torch.full((260, H, D), 0x1234, dtype=torch.int16, device=DEV)
    qt, ws = to_dev_bits(q), torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    got, owned = from_dev_bits(out), ~np.isnan(want[:, 0, 0])
    assert owned.sum() == 101 and (got[~owned] == 0x1234).all()
    _close(got[owned], want[owned], dev[owned])
    pool.close()


@FMT
def test_blocks_beyond_4_gib(fmt):
    """Block ids whose byte offsets pass 32 bits, signed and unsigned."""
    H, D = 40, 128
    bb = B.block_bytes(H, D, 16, R.FORMATS[fmt])
    blocks = (9 << 30) // bb
    far = torch.zeros(blocks * bb, dtype=torch.uint8, device=DEV).view(blocks, bb)
    rng = np.random.default_rng(3)
    batch = W.assemble_batch(H, D, 16, 16, [100, 90], [1, 40], rng)
    near = R.random_pool(batch, H, D, fmt, rng)
    where = np.linspace(0, blocks - 1, 16).astype(np.int32)      # small block -> far block
    far[torch.from_numpy(where.astype(np.int64)).to(DEV)] = torch.from_numpy(near).to(DEV)
    q = W.randn_bf16((41, H, D), rng)
    want, dev = R.attention(near, batch, q, H, fmt)
    tables = np.where(batch.block_tables >= 0, where[np.maximum(batch.block_tables, 0)], -1).astype(np.int32)
    pool = B.KvPool.from_tensor(far, H, D, dtype=R.FORMATS[fmt])
    desc = B.HostDesc(batch.ctx_len, batch.q_len, batch.q_start, tables, batch.scale)
    qt, out = to_dev_bits(q), torch.zeros((41, H, D), dtype=torch.int16, device=DEV)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    k, v = (torch.zeros((41, H, D), dtype=torch.int16, device=DEV) for _ in range(2))
    pool.kv_read_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    _close(from_dev_bits(out), want, dev)
    back = [R.context(near, batch, s, H, D, fmt)[0][-int(batch.q_len[s]):] for s in range(2)]
    assert np.array_equal(W.bf16_bits_to_f64(from_dev_bits(k)), np.concatenate(back))
    pool.kv_write_span(desc, k.data_ptr(), v.data_ptr())         # the same values again: nothing changes but the sign of zeros
    k2, v2 = (torch.zeros((41, H, D), dtype=torch.int16, device=DEV) for _ in range(2))
    pool.kv_read_span(desc, k2.data_ptr(), v2.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(k, k2) and torch.equal(v, v2)
    pool.close()


@FMT
def test_a_workspace_without_room_for_the_splits(fmt):
    H, D = 4, 128
    rng = np.random.default_rng(2)
    batch = W.assemble_batch(H, D, 16, 200, [2000, 300, 500], [1, 40, 200], rng)
    pool_bytes = R.random_pool(batch, H, D, fmt, rng)
    q = W.randn_bf16((241, H, D), rng)
    want = R.attention(pool_bytes, batch, q, H, fmt)
    pool, _ = _pool(pool_bytes, H, H, D, fmt)
    desc = B.HostDesc.from_batch(batch)
    full = pool.workspace_bytes(desc)
    pool.set_tuning(decode_part_tokens=4096, span_part_tokens=1 << 20)
    least = pool.workspace_bytes(desc)
    pool.set_tuning()
    assert least < full
    _close(_run(pool, batch, q, ws_bytes=least), *want)
    ws, qt = torch.empty(least, dtype=torch.uint8, device=DEV), to_dev_bits(q)
    assert pool.paged_attn_mixed(desc, qt.data_ptr(), qt.data_ptr(), ws.data_ptr(), 256, check=False) == B.IC_ESIZE
    pool.close()


# ------------------------------------------------------------------------------------------ used together
@FMT
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 128), (8, 2, 64), (2, 2, 256)])
def test_chunk_by_chunk_equals_one_shot(fmt, H, Hkv, D):
    """A context recomputed in chunks (write, then attention, every iteration) next to a request that decodes, from one plan per
    iteration over two layers; the cache is read back at the end."""
    rng = np.random.default_rng(21)
    n, chunks, L = 230, [100, 64, 3, 62, 1], 2
    table = rng.permutation(40).astype(np.int32)
    new = [[W.randn_bf16((n, Hkv, D), rng) for _ in range(2)] for _ in range(L)]
    qs = [W.randn_bf16((n, H, D), rng) for _ in range(L)]
    other = [W.randn_bf16((len(chunks), 2, Hkv, D), rng) for _ in range(L)]    # the decoding request's tokens
    start = rng.integers(0, 256, (40, B.block_bytes(Hkv, D, 16, R.FORMATS[fmt])), dtype=np.uint8)
    made = [_pool(start.copy(), H, Hkv, D, fmt) for _ in range(L)]
    host = [start.copy() for _ in range(L)]
    st = torch.cuda.Stream()
    done, outs = 0, [[], []]
    tables = np.full((2, 20), -1, dtype=np.int32)
    tables[0, :15], tables[1, :2] = table[:15], table[15:17]
    for it, c in enumerate(chunks):
        batch = W.Batch(H, D, 16, 40, np.array([done + c, it + 1], np.int32), np.array([c, 1], np.int32), np.array([0, c], np.int32), tables,
                        float(np.float32(D ** -0.5)), num_kv_heads=Hkv)
        desc = B.HostDesc.from_batch(batch)
        ws = torch.empty(made[0][0].workspace_bytes(desc), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        plan = made[0][0].plan_create(desc, ws.data_ptr(), ws.numel(), st.cuda_stream)
        keep = []
        for l in range(L):
            k, v = (np.concatenate([new[l][i][done:done + c], other[l][it:it + 1, i]]) for i in range(2))
            q = np.concatenate([qs[l][done:done + c], qs[l][it:it + 1]])
            R.write(host[l], batch, k, v, fmt)
            want, dev = R.attention(host[l], batch, q, Hkv, fmt)
            kt, vt, qt, out = to_dev_bits(k), to_dev_bits(v), to_dev_bits(q), torch.zeros((c + 1, H, D), dtype=torch.int16, device=DEV)
            torch.cuda.synchronize()
            made[l][0].kv_write_span_planned(plan, kt.data_ptr(), vt.data_ptr(), st.cuda_stream)
            made[l][0].paged_attn_planned(plan, qt.data_ptr(), out.data_ptr(), st.cuda_stream)
            keep.append((kt, vt, qt, out, want, dev))
        back = [[torch.zeros((c + 1, Hkv, D), dtype=torch.int16, device=DEV) for _ in range(2)] for _ in range(L)]
        torch.cuda.synchronize()
        for l in range(L):
            made[l][0].kv_read_span_planned(plan, back[l][0].data_ptr(), back[l][1].data_ptr(), st.cuda_stream)
        st.synchronize()
        for l, (kt, vt, qt, out, want, dev) in enumerate(keep):
            _close(from_dev_bits(out), want, dev)
            outs[l].append(from_dev_bits(out)[:c])
            for i in range(2):
                ctx = R.context(host[l], batch, 0, Hkv, D, fmt)[i][-c:]
                assert np.array_equal(W.bf16_bits_to_f64(from_dev_bits(back[l][i]))[:c], ctx)
        plan.close()
        done += c
    one = W.Batch(H, D, 16, 40, np.array([n], np.int32), np.array([n], np.int32), np.array([0], np.int32), tables[:1], float(np.float32(D ** -0.5)),
                  num_kv_heads=Hkv)
    for l in range(L):
        want, dev = R.attention(host[l], one, qs[l], Hkv, fmt)
        _close(np.concatenate(outs[l]), want, dev)
        _close(_run(made[l][0], one, qs[l]), want, dev)
        made[l][0].close()


@FMT
def test_plan_of_another_dtype_is_refused(fmt):
    H, D = 4, 128
    other = "int8" if fmt == "e4m3" else "e4m3"
    batch = W.assemble_batch(H, D, 16, 40, [100, 60], [1, 20], np.random.default_rng(1))
    desc = B.HostDesc.from_batch(batch)
    a, _ = _pool(R.empty_pool(40, H, D), H, H, D, fmt)
    b, _ = _pool(R.empty_pool(40, H, D), H, H, D, other)
    c = B.KvPool.from_tensor(torch.zeros((40, 2, H, 16, D), dtype=torch.int16, device=DEV), H, D)
    ws = torch.empty(max(p.workspace_bytes(desc) for p in (a, b, c)), dtype=torch.uint8, device=DEV)
    x, y, z = (torch.zeros((21, H, D), dtype=torch.int16, device=DEV) for _ in range(3))
    plan = a.plan_create(desc, ws.data_ptr(), ws.numel())
    for p in (b, c):
        assert p.paged_attn_planned(plan, x.data_ptr(), y.data_ptr(), check=False) == B.IC_EINVAL
        assert p.kv_write_span_planned(plan, x.data_ptr(), y.data_ptr(), check=False) == B.IC_EINVAL
        assert p.kv_read_span_planned(plan, x.data_ptr(), y.data_ptr(), check=False) == B.IC_EINVAL
    assert a.kv_read_span_planned(plan, x.data_ptr(), x.data_ptr(), check=False) == B.IC_EINVAL
    assert a.kv_read_span_planned(plan, x.data_ptr() + 2, y.data_ptr(), check=False) == B.IC_EALIGN
    assert a.kv_read_span_planned(plan, x.data_ptr(), 0, check=False) == B.IC_ENULL
    torch.cuda.synchronize()
    plan.close()
    for p in (a, b, c):
        p.close()


@FMT
def test_swap_moves_whole_blocks(fmt):
    """Gather, scatter and the layered swap to pinned memory keep an 8-bit context's bytes; what comes back answers the same."""
    H, D, L = 5, 64, 2
    rng = np.random.default_rng(31)
    batch = W.assemble_batch(H, D, 16, 30, [150], [1], rng)
    n = 10
    ids, to = batch.block_tables[0, :n].copy(), None
    to = np.setdiff1d(np.arange(30), ids)[:n].astype(np.int32)
    pools = [_pool(R.random_pool(batch, H, D, fmt, np.random.default_rng(40 + l)), H, H, D, fmt) for l in range(L)]
    host = [t.cpu().numpy() for _, t in pools]
    bb = pools[0][0].block_bytes
    q = W.randn_bf16((1, H, D), rng)
    first = [_run(p, batch, q) for p, _ in pools]
    pinned = torch.zeros(L * n * bb, dtype=torch.uint8, pin_memory=True)
    staging = torch.empty(B.LayerSwapper.staging_bytes(pools[0][0], L, n), dtype=torch.uint8, device=DEV)
    sw = B.LayerSwapper([p for p, _ in pools], n, staging.data_ptr(), staging.numel())
    sw.swap_out(ids, pinned.data_ptr(), n * bb)
    sw.sync()
    got = pinned.numpy().reshape(L, n, bb)
    for l in range(L):
        assert np.array_equal(got[l], host[l][ids])
    sw.swap_in(to, pinned.data_ptr(), n * bb)
    sw.sync()
    moved = W.Batch(H, D, 16, 30, batch.ctx_len, batch.q_len, batch.q_start, to[None, :].copy(), batch.scale, num_kv_heads=H)
    for l, (p, t) in enumerate(pools):
        assert np.array_equal(t.cpu().numpy()[to], host[l][ids])
        assert np.array_equal(_run(p, moved, q), first[l])
    st = torch.zeros(n * bb, dtype=torch.uint8, device=DEV)
    for pack in (pools[0][0].kv_pack_blocks, pools[0][0].kv_pack_blocks_static):
        st.zero_()
        torch.cuda.synchronize()
        pack(ids, st.data_ptr(), st.numel())
        torch.cuda.synchronize()
        assert np.array_equal(st.cpu().numpy().reshape(n, bb), host[0][ids])
    sw.close()
    for p, _ in pools:
        p.close()


@FMT
@pytest.mark.parametrize("tuning", [dict(), dict(row_launch=2), dict(decode_part_tokens=64, span_part_tokens=64)])
def test_planned_calls_in_a_captured_graph(fmt, tuning):
    """One layer's write, attention and read back as a graph: every replay gives what the eager calls give on the inputs it finds."""
    H, D = 4, 128
    rng = np.random.default_rng(51)
    batch = W.assemble_batch(H, D, 16, 150, [900, 300, 64, 500], [1, 100, 2, 1], rng)
    desc, rows = B.HostDesc.from_batch(batch), batch.total_q_rows
    start = R.random_pool(batch, H, D, fmt, rng)
    pool, t = _pool(start.copy(), H, H, D, fmt)
    pool.set_tuning(**tuning)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    q, k, v, out, kb, vb = (torch.zeros((rows, H, D), dtype=torch.int16, device=DEV) for _ in range(6))
    plan = pool.plan_create(desc, ws.data_ptr(), ws.numel(), 0)
    torch.cuda.synchronize()

    def calls(s):
        pool.kv_write_span_planned(plan, k.data_ptr(), v.data_ptr(), s)
        pool.paged_attn_planned(plan, q.data_ptr(), out.data_ptr(), s)
        pool.kv_read_span_planned(plan, kb.data_ptr(), vb.data_ptr(), s)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls(side.cuda_stream)                                  # first use outside the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        calls(torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        for x in (q, k, v):
            x.copy_(to_dev_bits(W.randn_bf16((rows, H, D), np.random.default_rng(60 + i)) if x is not q else W.randn_bf16((rows, H, D), rng)))
        for x in (out, kb, vb):
            x.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        a = [x.clone() for x in (out, kb, vb, t)]
        for x in (out, kb, vb):
            x.zero_()
        calls(0)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, (out, kb, vb, t)))
        host = start.copy()
        R.write(host, batch, from_dev_bits(k), from_dev_bits(v), fmt)
        _close(from_dev_bits(out), *R.attention(host, batch, from_dev_bits(q), H, fmt))
    plan.close()
    pool.close()


@FMT
def test_pools_on_two_streams_do_not_meet(fmt):
    H, D = 4, 128
    runs = []
    for i in range(2):
        rng = np.random.default_rng(70 + i)
        batch = W.assemble_batch(H, D, 16, 150, [900, 300, 500], [1, 100, 1], rng)
        pb = R.random_pool(batch, H, D, fmt, rng)
        q = W.randn_bf16((102, H, D), rng)
        pool, t = _pool(pb, H, H, D, fmt)
        desc = B.HostDesc.from_batch(batch)
        runs.append((pool, t, desc, to_dev_bits(q), torch.zeros((102, H, D), dtype=torch.int16, device=DEV),
                     torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV), torch.cuda.Stream(), R.attention(pb, batch, q, H, fmt)))
    torch.cuda.synchronize()
    for _ in range(20):
        for pool, _, desc, q, out, ws, st, _ in runs:
            pool.paged_attn_mixed(desc, q.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), st.cuda_stream)
    torch.cuda.synchronize()
    for pool, _, _, _, out, _, _, want in runs:
        _close(from_dev_bits(out), *want)
        pool.close()


@FMT
def test_more_row_items_than_one_grid_dimension(fmt):
    """33000 sequences of one token: the result is that token's value (weight 1), to the bit."""
    n, H, D = 33000, 2, 64
    bb = B.block_bytes(1, D, 16, R.FORMATS[fmt])
    pool = B.KvPool.from_tensor(torch.full((n, bb), 0xFF, dtype=torch.uint8, device=DEV), H, D, num_kv_heads=1, dtype=R.FORMATS[fmt])
    rng = np.random.default_rng(21)
    ids = rng.permutation(n).astype(np.int32)[:, None]
    ones, start = np.ones(n, np.int32), np.arange(n, dtype=np.int32)
    desc = B.HostDesc(ones, ones, start, ids, 0.125, n)
    k, v = (to_dev_bits(W.randn_bf16((n, 1, D), rng)) for _ in range(2))
    q, out, back = to_dev_bits(W.randn_bf16((n, H, D), rng)), torch.zeros((n, H, D), dtype=torch.int16, device=DEV), torch.zeros_like(v)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.kv_write_span(desc, k.data_ptr(), v.data_ptr())
    pool.paged_attn_mixed(desc, q.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    pool.kv_read_span(desc, k.data_ptr(), back.data_ptr())
    torch.cuda.synchronize()
    # (as numbers: a code of -0 comes out as 0)
    assert np.array_equal(W.bf16_bits_to_f64(from_dev_bits(out)), np.broadcast_to(W.bf16_bits_to_f64(from_dev_bits(back)), (n, H, D)))
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (8, 2, 128), (1, 1, 256)])
def test_query_rows_that_are_not_finite_stay_alone(fmt, H, Hkv, D):
    """Columns of one row item and rows of one tile: a query of NaN or infinities is the NaN of its own row and head only."""
    ctx, q_len = [300, 200, 70, 90, 33], [150, 1, 5, 64, 2]
    rng = np.random.default_rng(31)
    batch = W.assemble_batch(H, D, 16, 60, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    want, dev = R.attention(pool_bytes, batch, q, Hkv, fmt)
    bad = q.copy()
    for i, r in enumerate((3, 100, 149, 150, 153, 170, 219, 221)):
        bad[r, i % H, i::16] = (0x7FC0, 0x7F80, 0xFF80)[i % 3]   # NaN, inf, -inf
        want[r, i % H] = np.nan
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    for tuning in (dict(), dict(span_kernel=1), dict(span_part_tokens=64, decode_part_tokens=64), dict(row_launch=2)):
        pool.set_tuning(**tuning)
        got, fine = W.bf16_bits_to_f64(_run(pool, batch, bad)), ~np.isnan(want)
        assert np.isnan(got[~fine]).all()
        bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -8 + 1e-3) * dev + 1e-6
        assert (np.abs(got - want)[fine] <= bound[fine]).all()
    pool.close()


@FMT
def test_the_same_call_gives_the_same_bits(fmt):
    """Partitions end in any order; rows split inside the row kernel, by the merge kernel, and beside tiles."""
    rng = np.random.default_rng(41)
    for H, Hkv, D, ctx, q_len in [(8, 8, 128, [5000, 900], [1, 1]), (8, 2, 64, [4700, 3000], [3, 1]), (8, 1, 128, [2500, 4200, 3100], [300, 1, 2])]:
        batch = W.assemble_batch(H, D, 16, sum(ctx) // 16 + 8, ctx, q_len, rng, num_kv_heads=Hkv)
        pool, _ = _pool(R.random_pool(batch, Hkv, D, fmt, rng), H, Hkv, D, fmt)
        q = W.randn_bf16((sum(q_len), H, D), rng)
        for tuning in (dict(), dict(decode_part_tokens=128, span_part_tokens=512), dict(row_launch=2)):
            pool.set_tuning(**tuning)
            first = _run(pool, batch, q)
            for _ in range(6):
                assert np.array_equal(_run(pool, batch, q), first)
        pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(8, 8, 64), (8, 8, 128), (3, 3, 256), (5, 1, 128), (12, 2, 64), (24, 1, 128), (16, 2, 256)])
@pytest.mark.parametrize("tuning,items", [(dict(), 600), (dict(), 2100), (dict(row_launch=3), 2100), (dict(row_launch=2), 600)])
def test_short_rows_in_numbers(fmt, H, Hkv, D, tuning, items):
    """Rows of few keys, more than there are places for workgroups: a wave each.  Among them long rows, split ones, fresh and short chunks."""
    rng = np.random.default_rng(H + D)
    units = Hkv * (-(-(H // Hkv) // 16))
    n = items // units + 3                                       # (600: those of up to 256 keys are a wave's, 2100: of up to 512)
    ctx = list(rng.integers(1, 70, n)) + [1, 32, 33, 64, 65, 255, 256, 257, 400, 512, 513, 5000, 90, 300, 64, 70]
    q_len = [1] * (len(ctx) - 4) + [90, 200, 2, 3]
    blocks = sum(-(-int(c) // 16) for c in ctx) + 5
    batch = W.assemble_batch(H, D, 16, blocks, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    pool, _ = _pool(pool_bytes, H, Hkv, D, fmt)
    pool.set_tuning(**tuning)
    got = _run(pool, batch, q)
    want, dev = R.attention(pool_bytes, batch, q, Hkv, fmt)
    _close(got, want, dev)
    _close(got[:len(ctx) - 4], want[:len(ctx) - 4], dev[:len(ctx) - 4], weights=ROWS_ONLY)
    assert np.array_equal(got, _run(pool, batch, q))
    pool.close()
