"""Calls of the paged operators that their documentation allows, or that have to be refused, and that can go wrong in ways of their
own (references in 64 bits: tests/paged_util.py)."""
import ctypes

import numpy as np
import pytest
import torch

from tests import paged_util as pu
from tests import test_gpu_paged as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2603_09215_b200 import binding
    return binding


def ints(v, dtype=torch.int32):
    return torch.tensor(np.asarray(v), dtype=dtype, device="cuda")


BF, FP, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def test_tables_whose_rows_overlap_are_refused(B):
    """An expanded table, and one whose rows begin inside one another: there is no row of its own for every sequence.  Of a table of one
    row the stride says nothing."""
    n, blocks, page = 3, 4, 16
    kc = torch.zeros((8, 2, page, 64), dtype=FP, device="cuda")
    q, lens = torch.zeros((n, 4, 64), dtype=FP, device="cuda"), ints([40, 50, 64])
    flat = ints(range(7))
    for table in (flat[:blocks].view(1, blocks).expand(n, blocks), flat.as_strided((n, blocks), (1, 1))):
        out = torch.full_like(q, 7.0)
        ring, queue = ints(range(8)), ints([0, 8])
        for call in (lambda: B.paged_attention(q, kc, kc, table, lens, out=out),
                     lambda: B.page_map(lens, ints([1] * n), table, ring, queue, page, max_rows=8)):
            with pytest.raises(B.SparskError) as e:
                call()
            assert e.value.code == B.EINVAL
        torch.cuda.synchronize()
        assert (out == 7).all() and flat.tolist() == list(range(7)) and ring.tolist() == list(range(8))
        one = B.paged_attention(q[:1], kc, kc, table[:1], lens[:1])
        assert (one == 0).all()


@pytest.mark.parametrize("cache,hd", [(FP, 64), (FP, 128), (BF, 128), (E4, 64), (E4, 128)])
def test_what_lies_behind_every_end_is_cleared(B, cache, hd):
    """Hundreds of segments, each with an end inside a box of 16 positions behind which lie NaN: cleared by some of a warp's lanes,
    read by others.  Whatever lies there, the bits of the result are the same, every time."""
    n, hq, hk, page = 256, 8, 2, 16
    gen = torch.Generator("cuda").manual_seed(hd)
    lens = [1 + (i * 7) % 47 for i in range(n)]
    blocks = 3
    table = torch.randperm(n * blocks, generator=gen, device="cuda").to(torch.int32).view(n, blocks)
    kc, vc = (torch.randn((n * blocks, hk, page, hd), generator=gen, device="cuda") for _ in "kv")
    q = torch.randn((n, hq, hd), generator=gen, device="cuda").to(BF)
    behind = torch.arange(blocks * page, device="cuda")[None] >= ints(lens)[:, None]  # [sequence, position]
    place = (table.long()[:, :, None] * page + torch.arange(page, device="cuda")).view(n, -1)[behind]
    want = None
    for fill in (0.0, float("nan"), 3.0, float("nan")):
        for c in (kc, vc):
            c[place // page, :, place % page] = fill
        k8, v8 = kc.to(cache), vc.to(cache)
        for _ in range(5):
            got = B.paged_attention(q, k8, v8, table, ints(lens))
            want = got if want is None else want
            assert torch.equal(got, want) and not bool(got.isnan().any())


@pytest.mark.parametrize("gap", [9.0, 17.0, 20.0, 30.0, 60.0])
@pytest.mark.parametrize("qt,cache", base.TYPES)
def test_light_positions_behind_a_sink(B, qt, cache, gap):
    """The first position's score lies `gap` above the others', those of the next box half as far, and what both boxes hold is zero:
    the output is what the light positions say, however light.  (Nothing of the sink's box counts, so that every weight that does is off
    by its rounding, 2^-11, which base.check_attn allows, and 16 of them by 16 times 2^-20 of their largest.)"""
    lens, rows, page, hd = [3000, 40, 700, 33], [1, 2, 1, 1], 16, 64
    q, kc, vc, table, start, _ = base.attn_case(lens, rows, 8, 2, hd, page, qt, cache, "hnd", int(gap))
    q /= 4.0 if cache != E4 else 64.0  # (8-bit pages hold numbers sixteen times as large)
    q[..., 0] = gap / 64 * hd ** 0.5
    kc[..., 0] = torch.where(kc[..., 0].float().isnan(), kc[..., 0].float(), 0.0).to(cache)
    for i in range(len(lens)):
        first, second = (kc[int(table[i, b])] for b in (0, 1))
        first[:, 0] = 0.0
        first[:, 0, 0], second[:, 0, 0] = 64.0, 32.0
        vc[int(table[i, 0])], vc[int(table[i, 1])] = 0.0, 0.0
    base.check_attn(B, q, kc, vc, table, lens, start, [None, None], max_rows=2, max_len=3000)
    base.check_attn(B, q, kc, vc, table, lens, start, [None, None])


@pytest.mark.parametrize("lens,rows,hq,hk,hd,qt,cache,nth,hint", [
    ([20000], [1], 8, 2, 64, BF, FP, 40, 0),             # two segments cut into many shares: partials that are joined
    ([100] * 300, [1] * 300, 8, 2, 128, FP, FP, 7, 100),   # short segments, several to a share, none cut
    ([900, 4000, 33, 0, 2500] * 8, [4, 1, 3, 1, 2] * 8, 32, 2, 128, BF, E4, 100, 0),
    ([5], [1], 4, 2, 64, BF, BF, 1, 5),
])
def test_a_wait_that_runs_out(B, lens, rows, hq, hk, hd, qt, cache, nth, hint):
    """One CTA's stages wait for bytes that do not come (two seconds, and two more for the copies to have landed).  The call ends, its
    status says so, and every row is either what it always is or NaN; the next call is as if nothing had been."""
    q, kc, vc, table, start, _ = base.attn_case(lens, rows, hq, hk, hd, 16, qt, cache, "hnd", nth)
    L, t, n, s = B.load(), ints(table), ints(lens), ints(start)
    new = lambda: (torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 5.0, device="cuda"))  # noqa: E731
    status = ints([0])
    a = B.PagedAttnArgs()
    a.pool.k, a.pool.v = kc.data_ptr(), vc.data_ptr()
    a.pool.page_stride, a.pool.head_stride, a.pool.pos_stride = kc.stride()[:3]
    types = {BF: B.BF16, FP: B.FP16, E4: B.E4M3}
    a.pool.type, a.q_type = types[cache], types[qt]
    a.pool.n_pages, a.pool.n_kv_heads, a.pool.page_size, a.pool.head_dim = kc.shape
    a.q, a.block_table, a.seq_len, a.row_start = q.data_ptr(), t.data_ptr(), n.data_ptr(), s.data_ptr()
    a.table_stride, a.max_blocks = table.shape[1], table.shape[1]
    a.q_row_stride = a.out_row_stride = hq * hd
    a.q_head_stride = a.out_head_stride = hd
    a.n_rows, a.n_seqs, a.n_q_heads, a.max_len = len(q), len(lens), hq, hint
    nbytes = L.sparsk_paged_attention_scratch_bytes(ctypes.addressof(a))
    scratch = torch.full((nbytes,), 0x55, dtype=torch.uint8, device="cuda")

    def run(inject, with_status=True):
        out, lse = new()
        a.out, a.lse, a.status, a.inject_short_copy = out.data_ptr(), lse.data_ptr(), status.data_ptr() if with_status else None, inject
        assert L.sparsk_paged_attention(ctypes.addressof(a), scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream) == B.OK
        torch.cuda.synchronize()
        return out, lse

    want, want_lse = run(0)
    assert int(status) == 0 and not bool(want.isnan().any()) and not bool(want_lse.isnan().any())
    assert torch.equal(B.paged_attention(q, kc, vc, t, n, row_start=s, max_len=hint, status=status), want) and int(status) == 0
    got, got_lse = run(nth)
    assert int(status) == B.PAGED_TIMEOUT
    lost = got.isnan().all(-1)
    assert bool(lost.any()) and torch.equal(lost, got.isnan().any(-1)) and torch.equal(lost, got_lse.isnan())
    assert torch.equal(got[~lost], want[~lost]) and torch.equal(got_lse[~lost], want_lse[~lost])
    got, got_lse = run(0)
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse) and int(status) == B.PAGED_TIMEOUT  # (the caller clears it)
    if len(lens) == 1:
        status.zero_()
        assert bool(run(nth, with_status=False)[0].isnan().any()) and int(status) == 0


def test_a_scale_that_fp32_does_not_hold_is_refused(B):
    """Rounded to zero it would mean the default; the smallest that fp32 holds makes all weights equal."""
    q, kc, vc, table, start, _ = base.attn_case([20], [1], 4, 2, 64, 16, FP, FP, "hnd", 1)
    for scale in (1e-46, 1e-300, -1e-46):
        with pytest.raises(B.SparskError) as e:
            B.paged_attention(q, kc, vc, ints(table), ints([20]), scale=scale)
        assert e.value.code == B.EINVAL
    base.check_attn(B, q, kc, vc, table, [20], start, [None, None], scale=2e-38)


def test_no_page_is_lost_or_handed_out_twice(B):
    """Requests that come, grow and end for many steps, steps that are refused among them: after each, the pages of the live sequences
    and those of the queue are all pages, once each."""
    n, page, pages, blocks, most = 7, 4, 40, 12, 64
    rng = np.random.default_rng(3)
    table = torch.full((n, blocks), -1, dtype=torch.int32, device="cuda")
    ring = ints(np.concatenate([rng.permutation(pages), np.full(5, -1)]))
    size = len(ring)
    lens, queue, refused = ints([0] * n), ints([0, pages]), 0
    for step in range(120):
        rows = rng.integers(0, 7, n) - (rng.random(n) < 0.1) * 100
        rows = np.maximum(rows, -1)
        host = lens.tolist(), queue.tolist(), table.cpu().numpy(), ring.cpu().numpy()
        want = pu.page_map(host[0], rows, host[2], host[3], host[1], page, most)
        m = B.page_map(lens, ints(rows), table, ring, queue, page, max_rows=most)
        assert (int(m.status) == 0) == (want is not None)
        if want is None:
            refused += 1
            rows = np.where(rng.random(n) < 0.5, -1, 0)  # (room again)
            want = pu.page_map(host[0], rows, host[2], host[3], host[1], page, most)
            m = B.page_map(lens, ints(rows), table, ring, queue, page, max_rows=most)
            assert int(m.status) == 0
        lens, queue = m.seq_len, m.queue
        assert lens.tolist() == want[2].tolist() and queue.tolist() == want[3].tolist()
        t, r, (head, count) = table.tolist(), ring.tolist(), queue.tolist()
        held = [t[i][b] for i, length in enumerate(lens.tolist()) for b in range(-(-length // page))]
        assert sorted(held + [r[(head + k) % size] for k in range(count)]) == list(range(pages)), step
    assert refused > 5


@pytest.mark.parametrize("scale", [0.5, 4.0, 10.0])
@pytest.mark.parametrize("qt,cache", [(BF, FP), (FP, FP), (BF, E4), (FP, E4)])
def test_weights_are_right_to_what_is_promised(B, qt, cache, scale):
    """Scores far apart, every third position (the heaviest often among them) of zero values.  A weight may be off by its rounding,
    2^-11, and by 2^-20 of the largest of the same 16 positions; a score by the fp32 sums of its products; numbers below fp32's normal
    range are zero (2^-120 is far above what they can add up to)."""
    lens, rows, page, hd, hq, hk = [1500, 17, 100, 333], [1, 4, 9, 2], 32, 64, 8, 2
    q, kc, vc, table, start, _ = base.attn_case(lens, rows, hq, hk, hd, page, qt, cache, "nhd", 31)
    for i, length in enumerate(lens):
        for p in range(0, length, 3):
            vc[int(table[i, p // page]), :, p % page] = 0.0
    out = B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start), scale=scale).double().cpu().numpy()
    qd, kd, vd = (t.double().cpu().numpy() for t in (q, kc, vc))
    for i, (length, R) in enumerate(zip(lens, rows)):
        for j in range(R):
            p = np.arange(length - R + 1 + j)
            k, v = (x[table[i, p // page], :, p % page] for x in (kd, vd))  # [position, head, dim]
            first = np.arange(0, len(p), 16)
            for h in range(hq):
                kh, vh, x = k[:, h * hk // hq], v[:, h * hk // hq], qd[start[i] + j, h]
                s = scale * kh @ x
                w = np.exp(s - s.max())
                want = w @ vh / w.sum()
                d = scale * (np.abs(kh) @ np.abs(x)).max() * (hd + 8) * 2.0 ** -24 + 2.0 ** -20
                tol = (w @ np.abs(vh)) / w.sum() * (2.0 ** -11 + 2 * d + (len(p) + 64) * 2.0 ** -24)
                tol += 2.0 ** -20 * np.maximum.reduceat(w, first) @ np.add.reduceat(np.abs(vh), first) / w.sum() + 2.0 ** -120
                assert (np.abs(out[start[i] + j, h] - want) <= tol + pu.half_step(qt) * (np.abs(want) + tol) + pu.TINY[qt]).all(), (i, j, h)
