"""8-bit pools on the GPU at the ends of bf16's range.

Tolerances as in test_gpu_q8.py: half a step of the result (2^-8 of it), and the weights' errors times the mean distance of the values from
the result: 2^-8 for tiles, whose weights are rounded to bf16, and 1e-3 for what fp32 loses in the exponents."""
import numpy as np
import pytest
import torch

import q8_ref as R
from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W
from gpu_common import DEV, from_dev_bits, to_dev_bits

pytestmark = pytest.mark.gpu
FMT = pytest.mark.parametrize("fmt", ["e4m3", "int8"])
LARGEST = 0x7F7F                                                 # bits of the largest finite bf16 number, 255 * 2^120


def _lowered(codes, scales, fmt):
    """What the definition adds to rounding to nearest: a code that stands for 2^128, which bf16 does not hold, becomes the one below."""
    codes = codes.copy()
    with np.errstate(invalid="ignore"):
        over = np.abs(R.values(codes, scales, fmt)) >= 2.0 ** 128
    # ascending magnitudes are ascending codes; negative integers are two's complement
    down = np.where((codes >= 128) & (fmt == "int8"), codes + 1, codes - 1)
    codes[over] = down[over]
    return codes


def _write(pool_bytes, batch, k_bits, v_bits, fmt):
    """kv_write_span on the host, by the definition."""
    Hkv, D = k_bits.shape[1:]
    R.write(pool_bytes, batch, k_bits, v_bits, fmt)
    codes, scales = R.split(pool_bytes, Hkv, D)
    for s in range(batch.num_seqs):
        for t in range(int(batch.ctx_len[s] - batch.q_len[s]), int(batch.ctx_len[s])):
            b, slot = batch.block_tables[s, t // 16], t % 16
            for i in range(2):
                codes[b, i, :, slot] = _lowered(codes[b, i, :, slot], scales[b, :, i, slot], fmt)


@FMT
@pytest.mark.parametrize("H,D", [(1, 64), (3, 128), (2, 256)])
def test_a_finite_vector_is_kept_finite(fmt, H, D):
    """Every bf16 number from 192 * 2^120 to the largest, of both signs, alone and below a larger one in its vector."""
    n = 64
    rng = np.random.default_rng(D)
    batch = W.assemble_batch(H, D, 16, 12, [n], [n], rng)
    bits = rng.integers(0x7F00, 0x7F40, (2, n, H, D)) | (rng.integers(0, 2, (2, n, H, D)) << 15)
    for r in range(n):
        bits[:, r, :, 1::2] &= 0x8000                            # zeros, and
        bits[:, r, :, 0] = 0x7F40 + r                            # ... the vector's largest
        bits[:, r, :, 2] = 0x8000 | (0x7F40 + r)
        bits[:, r, :, 4] = 0x7F40 + max(0, r - 1)
    new = bits.astype(np.uint16)
    want = R.empty_pool(12, H, D)
    _write(want, batch, new[0], new[1], fmt)
    t = torch.from_numpy(R.empty_pool(12, H, D)).to(DEV)
    pool = B.KvPool.from_tensor(t, H, D, dtype=R.FORMATS[fmt])
    desc = B.HostDesc.from_batch(batch)
    k, v = to_dev_bits(new[0]), to_dev_bits(new[1])
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    pool.kv_write_span(desc, k.data_ptr(), v.data_ptr())
    pool.kv_read_span(desc, kb.data_ptr(), vb.data_ptr())
    torch.cuda.synchronize()
    gc, gs = R.split(t.cpu().numpy(), H, D)
    wc, ws = R.split(want, H, D)
    assert np.array_equal(gs, ws)
    assert np.array_equal(R.code_values(fmt)[gc], R.code_values(fmt)[wc], equal_nan=True)
    for got, x, kept in zip((kb, vb), new, R.context(want, batch, 0, H, D, fmt)):
        back, x = W.bf16_bits_to_f64(from_dev_bits(got)), W.bf16_bits_to_f64(x)
        assert np.isfinite(back).all() and np.array_equal(back, kept)
        # half a step, except where that is infinity: there 15 of 255 (e4m3) and three quarters of a step (integers)
        half = np.abs(x) * 2.0 ** -4 + 2.0 ** 104 if fmt == "e4m3" else np.where(np.abs(x) >= 63.5 * 2.0 ** 122, 0.75, 0.5) * 2.0 ** 122
        assert (np.abs(back - x) <= half).all()
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (2, 2, 128), (8, 2, 128), (1, 1, 256)])
@pytest.mark.parametrize("tuning", [dict(), dict(span_kernel=1), dict(span_kernel=2), dict(span_part_tokens=64, decode_part_tokens=64), dict(row_launch=2)])
def test_the_largest_number_in_a_value_shows_in_its_own_dimension(fmt, H, Hkv, D, tuning):
    """A value with the largest bf16 number at a position that earlier rows of its tile do not see: those rows are the 64-bit result, and
    of the later ones every dimension but that one (where fp32 sums of such numbers may overflow)."""
    n, at = 200, [70, 131, 199]
    rng = np.random.default_rng(H + D)
    batch = W.assemble_batch(H, D, 16, 40, [n, 90], [n, 1], rng, num_kv_heads=Hkv)
    k, v, q = W.randn_bf16((n + 1, Hkv, D), rng), W.randn_bf16((n + 1, Hkv, D), rng), W.randn_bf16((n + 1, H, D), rng)
    for i, t in enumerate(at):
        v[t] &= 0x8000                                           # (the scale of such a vector leaves nothing of smaller numbers)
        v[t, :, 7] = LARGEST if i % 2 else 0x8000 | LARGEST
    start = R.random_pool(batch, Hkv, D, fmt, rng)
    host = start.copy()
    _write(host, batch, k, v, fmt)
    t = torch.from_numpy(start).to(DEV)
    pool = B.KvPool.from_tensor(t, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    pool.set_tuning(**tuning)
    desc = B.HostDesc.from_batch(batch)
    kt, vt, qt, out = to_dev_bits(k), to_dev_bits(v), to_dev_bits(q), torch.zeros((n + 1, H, D), dtype=torch.int16, device=DEV)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.kv_write_span(desc, kt.data_ptr(), vt.data_ptr())
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    got = W.bf16_bits_to_f64(from_dev_bits(out))
    want, dev = R.attention(host, batch, q, Hkv, fmt)
    mine = np.ones((n + 1, H, D), dtype=bool)
    mine[at[0]:n, :, 7] = False
    bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -8 + 1e-3) * dev + 1e-6
    assert np.isfinite(got[mine]).all()
    assert (np.abs(got - want)[mine] <= bound[mine]).all()
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (8, 2, 128), (1, 1, 256)])
@pytest.mark.parametrize("tuning", [dict(), dict(span_kernel=1)])
def test_the_largest_number_in_a_key_meets_zeros(fmt, H, Hkv, D, tuning):
    """Keys with the largest bf16 number in a dimension where every query is 0: a finite product, 0."""
    n = 150
    rng = np.random.default_rng(H * D)
    batch = W.assemble_batch(H, D, 16, 40, [n, 90], [n, 1], rng, num_kv_heads=Hkv)
    k, v, q = W.randn_bf16((n + 1, Hkv, D), rng), W.randn_bf16((n + 1, Hkv, D), rng), W.randn_bf16((n + 1, H, D), rng)
    k[::13, :, 9] = LARGEST
    q[:, :, 9] = 0
    start = R.random_pool(batch, Hkv, D, fmt, rng)
    host = start.copy()
    _write(host, batch, k, v, fmt)
    t = torch.from_numpy(start).to(DEV)
    pool = B.KvPool.from_tensor(t, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    pool.set_tuning(**tuning)
    desc = B.HostDesc.from_batch(batch)
    kt, vt, qt, out = to_dev_bits(k), to_dev_bits(v), to_dev_bits(q), torch.zeros((n + 1, H, D), dtype=torch.int16, device=DEV)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.kv_write_span(desc, kt.data_ptr(), vt.data_ptr())
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    want, dev = R.attention(host, batch, q, Hkv, fmt)
    got = W.bf16_bits_to_f64(from_dev_bits(out))
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -8 + 1e-3) * dev + 1e-6).all()
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (2, 2, 128), (16, 1, 128), (1, 1, 256)])
@pytest.mark.parametrize("tuning", [dict(), dict(decode_part_tokens=192), dict(row_launch=3)])
def test_a_weight_ahead_of_the_running_maximum_meets_the_largest_scale(fmt, H, Hkv, D, tuning):
    """A key that scores 2^7.9 times the ones before it, by less than the running maximum's slack may be: its weight times the scale of a value
    with the largest bf16 number stays finite, and the dimensions where that value is 0 are the 64-bit result."""
    ctx = [150, 300, 170, 190]
    q_len = [1, 1, 3, 1]
    rng = np.random.default_rng(3)
    batch = W.assemble_batch(H, D, 16, 60, ctx, q_len, rng, num_kv_heads=Hkv)
    batch.scale = 1.0
    whole = W.Batch(H, D, 16, 60, batch.ctx_len, batch.ctx_len, np.cumsum([0] + ctx[:-1]).astype(np.int32), batch.block_tables, 1.0, num_kv_heads=Hkv)
    k, v = np.zeros((sum(ctx), Hkv, D), np.uint16), W.randn_bf16((sum(ctx), Hkv, D), rng)
    for s, c in enumerate(ctx):
        r = int(whole.q_start[s]) + 133                          # the fifth tile of 32 keys: the first wave has the first tile and this one
        k[r, :, 0] = W.f32_to_bf16_bits(np.float32(5.5))         # 7.93 in powers of two
        v[r] &= 0x8000
        v[r, :, 7] = LARGEST
    q = W.randn_bf16((sum(q_len), H, D), rng)
    q[:, :, 0] = W.f32_to_bf16_bits(np.float32(1.0))
    start = R.empty_pool(60, Hkv, D)
    host = start.copy()
    _write(host, whole, k, v, fmt)
    t = torch.from_numpy(start).to(DEV)
    pool = B.KvPool.from_tensor(t, H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    kt, vt, qt, out = to_dev_bits(k), to_dev_bits(v), to_dev_bits(q), torch.zeros(q.shape, dtype=torch.int16, device=DEV)
    pool.kv_write_span(B.HostDesc.from_batch(whole), kt.data_ptr(), vt.data_ptr())
    pool.set_tuning(**tuning)
    desc = B.HostDesc.from_batch(batch)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    got = W.bf16_bits_to_f64(from_dev_bits(out))
    want, dev = R.attention(host, batch, q, Hkv, fmt)
    others = np.arange(D) != 7
    got, want, dev = got[..., others], want[..., others], dev[..., others]
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= (2.0 ** -8 + 1e-5) * np.abs(want) + 1e-3 * dev + 1e-6).all()
    pool.close()


def _with_nan_vectors(pool_bytes, batch, H, Hkv, D, which, at, want):
    """A key (which 0) or a value (1) of K/V head 0 that is not finite at position at[s] of sequence s, and NaN in want where it shows."""
    codes, scales = R.split(pool_bytes, Hkv, D)
    for s, t in at.items():
        b, n, c = batch.block_tables[s, t // 16], int(batch.q_len[s]), int(batch.ctx_len[s])
        codes[b, which, 0, t % 16] = 0
        scales[b, 0, which, t % 16] = 255
        first = max(0, t - (c - n))
        want[batch.q_start[s] + first:batch.q_start[s] + n, :H // Hkv] = np.nan


def _shows_where_it_should(got_bits, want, dev):
    got, hit = W.bf16_bits_to_f64(got_bits), np.isnan(want)
    assert np.isnan(got[hit]).all()
    bound = (2.0 ** -8 + 1e-5) * np.abs(want) + (2.0 ** -8 + 1e-3) * dev + 1e-6
    assert (np.abs(got - want)[~hit] <= bound[~hit]).all()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 64), (2, 2, 128), (8, 2, 128), (1, 1, 256)])
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("row_launch", [2, 3])
def test_nan_vectors_in_the_rows_that_run_beside_tiles(fmt, H, Hkv, D, which, row_launch):
    ctx, q_len = [300, 200, 70, 90, 260], [200, 1, 20, 64, 1]
    at = {0: 211, 1: 37, 2: 61, 3: 40}                           # (the last sequence has none)
    rng = np.random.default_rng(6)
    batch = W.assemble_batch(H, D, 16, 70, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    want, dev = R.attention(pool_bytes, batch, q, Hkv, fmt)
    _with_nan_vectors(pool_bytes, batch, H, Hkv, D, which, at, want)
    pool = B.KvPool.from_tensor(torch.from_numpy(pool_bytes).to(DEV), H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    pool.set_tuning(row_launch=row_launch)
    desc = B.HostDesc.from_batch(batch)
    qt, out = to_dev_bits(q), torch.zeros(q.shape, dtype=torch.int16, device=DEV)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    _shows_where_it_should(from_dev_bits(out), want, dev)
    pool.close()


@FMT
@pytest.mark.parametrize("H,Hkv,D", [(8, 8, 64), (8, 8, 128), (3, 3, 256), (24, 2, 128)])
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("row_launch", [0, 2, 3])
def test_nan_vectors_in_rows_that_are_a_wave_each(fmt, H, Hkv, D, which, row_launch):
    """Short rows in numbers, every fifth with a vector that is not finite, its neighbours in the same workgroup without; fresh and short chunks."""
    rng = np.random.default_rng(H + D)
    n = 2 * 2100 // (Hkv * (-(-(H // Hkv) // 16))) // 2 + 3      # more than four times the places
    ctx = list(rng.integers(1, 70, n)) + [90, 300, 64, 70]
    q_len = [1] * n + [90, 200, 2, 3]
    at = {s: int(rng.integers(0, ctx[s])) for s in list(range(0, n, 5)) + [n, n + 2]}
    batch = W.assemble_batch(H, D, 16, sum(-(-int(c) // 16) for c in ctx) + 5, ctx, q_len, rng, num_kv_heads=Hkv)
    pool_bytes = R.random_pool(batch, Hkv, D, fmt, rng)
    q = W.randn_bf16((sum(q_len), H, D), rng)
    want, dev = R.attention(pool_bytes, batch, q, Hkv, fmt)
    _with_nan_vectors(pool_bytes, batch, H, Hkv, D, which, at, want)
    pool = B.KvPool.from_tensor(torch.from_numpy(pool_bytes).to(DEV), H, D, num_kv_heads=Hkv, dtype=R.FORMATS[fmt])
    pool.set_tuning(row_launch=row_launch)
    desc = B.HostDesc.from_batch(batch)
    qt, out = to_dev_bits(q), torch.zeros(q.shape, dtype=torch.int16, device=DEV)
    ws = torch.empty(pool.workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    pool.paged_attn_mixed(desc, qt.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    _shows_where_it_should(from_dev_bits(out), want, dev)
    pool.close()


@FMT
def test_a_context_moved_to_the_other_dtype_is_quantised_anew(fmt):
    """The cache there is the definition's of the values here: integers keep less of small numbers than e4m3, e4m3 less of large ones."""
    H, D = 3, 128
    other = "int8" if fmt == "e4m3" else "e4m3"
    rng = np.random.default_rng(15)
    batch = W.assemble_batch(H, D, 16, 30, [200, 16, 90], [200, 16, 90], rng)
    desc, src = B.HostDesc.from_batch(batch), R.random_pool(batch, H, D, fmt, rng)
    a = B.KvPool.from_tensor(torch.from_numpy(src).to(DEV), H, D, dtype=R.FORMATS[fmt])
    t = torch.from_numpy(R.empty_pool(30, H, D)).to(DEV)
    b = B.KvPool.from_tensor(t, H, D, dtype=R.FORMATS[other])
    k, v = (torch.zeros((batch.total_q_rows, H, D), dtype=torch.int16, device=DEV) for _ in range(2))
    a.kv_read_span(desc, k.data_ptr(), v.data_ptr())
    b.kv_write_span(desc, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    want = R.empty_pool(30, H, D)
    _write(want, batch, from_dev_bits(k), from_dev_bits(v), other)
    got, lost = t.cpu().numpy(), 0
    for s in range(batch.num_seqs):
        here = R.context(src, batch, s, H, D, fmt)
        for x, y, z in zip(here, R.context(got, batch, s, H, D, other), R.context(want, batch, s, H, D, other)):
            assert np.array_equal(y, z)
            lost += (x != y).sum()
    assert lost > 0
    a.close()
    b.close()
