"""The paged operators against references in 64 bits (tests/paged_util.py), each at the sizes and contents where it can go
wrong, and a serving loop that uses them one after another."""
import numpy as np
import pytest
import torch

from tests import paged_util as pu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2603_09215_b200 import binding
    return binding


def ints(v, dtype=torch.int32):
    return torch.tensor(np.asarray(v), dtype=dtype, device="cuda")


# ------------------------------------------------------------------ page map
def map_case(lens, rows, page, seed, spare=5, room=None, ring_size=None, max_rows=None):
    rng = np.random.default_rng(seed)
    had = [-(-n // page) for n in lens]
    has = [-(-(n + max(r, 0)) // page) for n, r in zip(lens, rows)]
    need = sum(max(0, b - a) for a, b in zip(had, has))
    pages = sum(had) + max(need + spare, 0)
    ring_size = ring_size or max(pages, 1)
    perm = rng.permutation(pages)
    table = np.full((len(lens), room or max(has + had + [1]) + 1), -7)
    at = 0
    for i, b in enumerate(had):
        b = min(b, table.shape[1])
        table[i, :b] = perm[at:at + b]
        at += b
    head, free = int(rng.integers(ring_size)), pages - at
    ring = np.full(ring_size, -9)
    ring[(head + np.arange(free)) % ring_size] = perm[at:]
    return table, ring, [head, free], max_rows if max_rows is not None else sum(max(r, 0) for r in rows) + 3


MAPS = [
    ([0], [1], 16), ([0], [0], 16), ([15], [1], 16), ([16], [1], 16), ([5], [-1], 4), ([0], [-1], 4),
    ([31, 32, 33, 0, 64], [1, 1, 1, 70, -1], 32),
    ([0] * 40, list(range(40)), 1), ([7, 0, 100, 3], [0, 0, 0, 0], 8),
    ([100, 90, 80], [-1, -1, -1], 16),
    ([(i * 37) % 500 for i in range(1500)], [1 if i % 11 else -1 for i in range(1500)], 48),
    ([(i * 37) % 90 for i in range(3001)], [(i * i) % 23 - 1 for i in range(3001)], 16),
    ([0, 5], [30000, 3], 128),
]


@pytest.mark.parametrize("lens,rows,page", MAPS)
def test_page_map(B, lens, rows, page):
    table, ring, queue, max_rows = map_case(lens, rows, page, len(lens))
    ref = pu.page_map(lens, rows, table, ring, queue, page, max_rows)
    dt, dr, dl = ints(table), ints(ring), ints(lens)
    m = B.page_map(dl, ints(rows), dt, dr, ints(queue), page, max_rows=max_rows)
    got = (dt, dr, m.seq_len, m.queue, m.row_start, m.row_seq, m.row_pos, m.slot_map)
    assert int(m.status) == 0
    for g, r, what in zip(got, ref, ("table", "ring", "seq_len", "queue", "row_start", "row_seq", "row_pos", "slot_map")):
        assert np.array_equal(g.cpu().numpy(), r), what
    assert np.array_equal(dl.cpu().numpy(), lens)


@pytest.mark.parametrize("what,code", [("short", 1), ("table", 2), ("rows", 4), ("length", 8), ("count", 8), ("queue", 8), ("ring", 8)])
def test_page_map_is_all_or_nothing(B, what, code):
    lens, rows, page = [40, 3, 64, 9], [30, 100, -1, 2], 16
    kw = {"short": dict(spare=-1), "table": dict(room=5), "rows": dict(max_rows=131), "ring": dict()}.get(what, {})
    table, ring, queue, max_rows = map_case(lens, rows, page, 1, **kw)
    if what == "length":
        lens[1] = -1
    if what == "count":
        rows[1] = -2
    if what == "queue":
        queue[0] = len(ring)
    if what == "ring":  # the ended sequence's pages do not fit behind the queue's own
        queue[1] = len(ring) - 3
    dt, dr = ints(table), ints(ring)
    m = B.page_map(ints(lens), ints(rows), dt, dr, ints(queue), page, max_rows=max_rows)
    assert int(m.status) == code
    assert np.array_equal(dt.cpu().numpy(), table) and np.array_equal(dr.cpu().numpy(), ring)
    assert m.seq_len.tolist() == lens and m.queue.tolist() == queue and m.row_start.tolist() == [0] * 5
    assert m.row_seq.tolist() == m.row_pos.tolist() == m.slot_map.tolist() == [-1] * max_rows


def test_page_map_lengths_beyond_32_bits(B):
    """Sums of lengths and rows near 2^31 are told apart from small ones."""
    big = 2 ** 31 - 1
    t, r = ints(np.zeros((3, 4))), ints(np.arange(8))
    for rows, code in (([big, big, 2], 2), ([0, 0, big], 2)):
        m = B.page_map(ints([0, 0, 5]), ints(rows), t, r, ints([0, 8]), 16, max_rows=4)
        assert int(m.status) == code
    m = B.page_map(ints([0, 0, 0]), ints([2 ** 30] * 3), ints(np.zeros((3, 4))), r, ints([0, 8]), 2 ** 29, max_rows=4)
    assert int(m.status) == 4  # 6 pages of 8, but 3 * 2^30 rows


def test_page_map_table_rows_apart(B):
    """A table that is part of a wider one."""
    table, ring, queue, max_rows = map_case([20, 0], [30, 9], 16, 3)
    ref = pu.page_map([20, 0], [30, 9], table, ring, queue, 16, max_rows)
    widest = torch.full((2, table.shape[1] + 5), 55, dtype=torch.int32, device="cuda")
    part = widest[:, 2:2 + table.shape[1]]
    part.copy_(ints(table))
    m = B.page_map(ints([20, 0]), ints([30, 9]), part, ints(ring), ints(queue), 16, max_rows=max_rows)
    assert np.array_equal(part.cpu().numpy(), ref[0]) and np.array_equal(m.slot_map.cpu().numpy(), ref[7])
    assert bool((widest[:, :2] == 55).all()) and bool((widest[:, 2 + table.shape[1]:] == 55).all())


# ------------------------------------------------------------------ rows into pages
def pool_of(pages, heads, page, hd, dtype, layout, gen):
    shape = (pages, heads, page, hd) if layout == "hnd" else (pages, page, heads, hd)
    x = torch.randn(shape, generator=gen, device="cuda")
    x = (x * 16 if dtype == torch.float8_e4m3fn else x).to(dtype)
    return x if layout == "hnd" else x.transpose(1, 2)


def turned(x, cs):
    """(turned, sum of the two products' magnitudes), float64."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cs[:, None, :, 0], cs[:, None, :, 1]
    return (np.concatenate([a * c - b * s, b * c + a * s], -1),
            np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], -1))


def near(got, want, dtype, slack):
    """Half a step of the type, and `slack` for the arithmetic before it."""
    w = np.clip(want, -pu.MAX[dtype], pu.MAX[dtype]) if dtype in pu.MAX else want
    tol = pu.half_step(dtype) * (np.abs(w) + slack) + slack + pu.TINY[dtype]
    return (np.abs(got - w) <= tol) | (np.isnan(got) & np.isnan(w))


@pytest.mark.parametrize("n,hq,hk,hd,page,x,cache,layout,turn", [
    (1, 4, 2, 64, 16, torch.bfloat16, torch.float16, "hnd", True),
    (7, 28, 4, 128, 16, torch.bfloat16, torch.float16, "nhd", True),
    (33, 3, 1, 64, 5, torch.float32, torch.bfloat16, "hnd", True),
    (129, 8, 8, 128, 64, torch.float16, torch.float8_e4m3fn, "nhd", True),
    (64, 0, 3, 64, 48, torch.float32, torch.float8_e4m3fn, "hnd", False),
    (515, 5, 5, 128, 1, torch.float16, torch.bfloat16, "hnd", False),
    (20, 2, 2, 128, 32, torch.float32, torch.float16, "nhd", True),
])
@pytest.mark.parametrize("shift", [0, 1])
def test_append(B, n, hq, hk, hd, page, x, cache, layout, turn, shift):
    """Strided slices of one product's rows (shift: that start where no 16-byte access can), left-out rows, other slots untouched."""
    gen = torch.Generator("cuda").manual_seed(n * 7 + hk)
    pages = -(-n // page) + 3
    width = (hq + 2 * hk) * hd
    buf = torch.randn(n * (width + 8 * shift) + 8, generator=gen, device="cuda").to(x)
    if x == torch.float32:
        buf[5:9] = torch.tensor([7e4, -7e4, 500.0, -1e6])
    full = buf[shift:shift + n * (width + 8 * shift)].view(n, -1)[:, :width].view(n, hq + 2 * hk, hd)
    q, k, v = full[:, :hq], full[:, hq:hq + hk], full[:, hq + hk:]
    kc, vc = (pool_of(pages, hk, page, hd, cache, layout, gen) for _ in "kv")
    before = [t.double().cpu().numpy() for t in (kc, vc)]
    slots = torch.randperm(pages * page, generator=gen, device="cuda")[:n]
    slots[n // 2:n // 2 + 1] = -1
    if n > 20:
        slots[3] = pages * page + 2
    length = 97
    pos = torch.randint(0, length, (n,), generator=gen, device="cuda").to(torch.int32)
    rope = torch.randn((length, hd // 2, 2), generator=gen, device="cuda") if turn else None
    if turn and n > 20:
        pos[5], pos[6] = -1, length
    scales = [torch.rand(hk, generator=gen, device="cuda") + 0.01 for _ in "kv"] if cache == torch.float8_e4m3fn else [None, None]
    qo_type = torch.float16 if x == torch.float16 else torch.bfloat16
    q_out = torch.full((n, hq, hd), 3.0, dtype=qo_type, device="cuda") if hq else None
    B.paged_append(k, v, kc, vc, slots, q=q if hq else None, q_out=q_out, row_pos=pos if turn else None, rope=rope, k_scale=scales[0],
                   v_scale=scales[1])
    sl, ps = slots.cpu().numpy(), pos.cpu().numpy()
    on = (ps >= 0) & (ps < length) if turn else np.ones(n, bool)
    cs = rope.double().cpu().numpy()[np.clip(ps, 0, length - 1)] if turn else None
    dbl = lambda t: t.double().cpu().numpy()  # noqa: E731
    kt, kslack = turned(dbl(k), cs) if turn else (dbl(k), np.zeros(k.shape))
    for got, old, new, slack, scale in ((kc, before[0], kt, kslack, scales[0]), (vc, before[1], dbl(v), np.zeros(v.shape), scales[1])):
        got = dbl(got)
        s = 1.0 if scale is None else dbl(scale)[:, None]
        stay = (sl >= 0) & (sl < pages * page) & on
        at = sl[stay]
        # two products, a sum and a quotient in fp32: four roundings of at most the products' magnitudes
        assert near(got[at // page, :, at % page], (new / s)[stay], cache, 4 * 2.0 ** -24 * ((slack + np.abs(new)) / s)[stay]).all()
        old[at // page, :, at % page] = got[at // page, :, at % page]
        assert np.array_equal(old, got)
    if hq:
        qt, slack = turned(dbl(q), cs) if turn else (dbl(q), np.zeros(q.shape))
        got = dbl(q_out)
        assert near(got[on], qt[on], qo_type, 3 * 2.0 ** -24 * slack[on]).all() and (got[~on] == 3.0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shift", range(8))
def test_append_rows_at_every_offset(B, dtype, shift):
    """Rows that start at any number of a 16-byte block, the last one at its memory's end: the same as from aligned rows."""
    n, hq, hk, hd, page = 9, 3, 2, 64, 16
    gen = torch.Generator("cuda").manual_seed(shift)
    w = (hq + 2 * hk) * hd
    x = torch.randn((n, w), generator=gen, device="cuda").to(dtype)
    for gap in (0, 1, 8):
        flat = torch.full((shift + n * (w + gap) - gap,), float("nan"), dtype=dtype, device="cuda")
        rows = flat.as_strided((n, w), (w + gap, 1), shift)
        rows.copy_(x)
        got = []
        for y in (x, rows):
            q, k, v = (t.unflatten(1, (-1, hd)) for t in (y[:, :hq * hd], y[:, hq * hd:(hq + hk) * hd], y[:, (hq + hk) * hd:]))
            kc, vc = (torch.zeros((2, hk, page, hd), dtype=FP, device="cuda") for _ in range(2))
            out = B.paged_append(k, v, kc, vc, ints(range(n), torch.int64), q=q, row_pos=ints(range(n)),
                                 rope=torch.arange(n * hd, dtype=torch.float32, device="cuda").view(n, hd // 2, 2) / 100)
            got.append((out, kc, vc))
        assert all(torch.equal(a, b) and not a.isnan().any() for a, b in zip(*got))


def test_append_not_finite_and_in_place(B):
    gen = torch.Generator("cuda").manual_seed(0)
    for cache in (torch.float16, torch.bfloat16, torch.float8_e4m3fn):
        kc, vc = (pool_of(2, 1, 16, 64, cache, "hnd", gen) for _ in "kv")
        k = torch.zeros((1, 1, 64), device="cuda")
        k[0, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
        B.paged_append(k, -k, kc, vc, ints([17], torch.int64))
        got = kc[1, 0, 1, :4].float().tolist()
        most = pu.MAX.get(cache, float("inf"))
        assert got[0] != got[0] and got[1:] == [most, -most, 0.0], (cache, got)
    # queries turned where they are
    q = torch.randn((5, 3, 64), generator=gen, device="cuda").to(torch.bfloat16)
    rope = torch.randn((9, 32, 2), generator=gen, device="cuda")
    pos, k = ints([0, 8, 3, 3, 1]), torch.zeros((5, 1, 64), dtype=torch.bfloat16, device="cuda")
    kc, vc = (pool_of(1, 1, 16, 64, torch.float16, "hnd", gen) for _ in "kv")
    slots = ints([0, 1, 2, 3, 4], torch.int64)
    want = B.paged_append(k, k, kc, vc, slots, q=q, row_pos=pos, rope=rope)
    assert want.data_ptr() != q.data_ptr()
    B.paged_append(k, k, kc, vc, slots, q=q, q_out=q, row_pos=pos, rope=rope)
    assert torch.equal(q, want)


def test_append_beyond_4_gib(B):
    """A pool of more than 2^32 bytes: offsets are 64 bits wide."""
    pages, page = 33000, 16
    kc, vc = (torch.zeros((pages, 64, page, 128), dtype=torch.float8_e4m3fn, device="cuda") for _ in "kv")
    k = torch.ones((2, 64, 128), dtype=torch.bfloat16, device="cuda")
    B.paged_append(k, 2 * k, kc, vc, ints([pages * page - 1, 7], torch.int64))
    assert float(kc[-1, :, -1].float().min()) == 1.0 and float(vc[-1, :, -1].float().min()) == 2.0
    assert float(kc[0, :, 7].float().min()) == 1.0 and int(kc.view(torch.uint8).count_nonzero()) == 2 * 64 * 128


# ------------------------------------------------------------------ attention over pages
def attn_case(lens, rows, hq, hk, hd, page, qt, cache, layout, seed, scales=False):
    gen = torch.Generator("cuda").manual_seed(seed)
    blocks = [-(-max(n, 0) // page) for n in lens]
    pages = sum(blocks) + 4
    perm = torch.randperm(pages, generator=gen, device="cuda").cpu().numpy()
    table = np.full((len(lens), max(blocks + [0]) + 2), -1)
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = perm[at:at + b]
        at += b
    start = np.concatenate([[0], np.cumsum(rows)]).astype(int)
    q = torch.randn((int(start[-1]), hq, hd), generator=gen, device="cuda").to(qt)
    kc, vc = (pool_of(pages, hk, page, hd, cache, layout, gen) for _ in "kv")
    # what no row may look at: behind the sequences' ends and in pages of nobody
    for i, n in enumerate(lens):
        if n > 0 and n % page:
            for c in (kc, vc):
                c[int(table[i, n // page]), :, n % page:] = float("nan")
    for p in perm[at:]:
        kc[int(p)], vc[int(p)] = float("nan"), float("nan")
    sc = [torch.rand(hk, generator=gen, device="cuda") * 0.05 + 0.04 for _ in "kv"] if scales else [None, None]
    return q, kc, vc, table, start, sc


def check_attn(B, q, kc, vc, table, lens, start, sc, scale=0.0, **kw):
    n, hq, hd = q.shape
    out = torch.full((n + 2, hq, hd), 5.0, dtype=q.dtype, device="cuda")
    lse = torch.full((n, hq), 5.0, device="cuda")
    B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start), out=out[:n], lse=lse, k_scale=sc[0], v_scale=sc[1],
                      scale=scale, **kw)
    dbl = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    want, wl, tol, ltol = pu.attend(dbl(q), dbl(kc), dbl(vc), table, lens, start, scale or hd ** -0.5, 2.0 ** -11, dbl(sc[0]), dbl(sc[1]))
    got, gl = dbl(out), dbl(lse)
    assert (got[n:] == 5.0).all()
    for r in range(n):
        if want[r] is None:
            assert (got[r] == 5.0).all() and (gl[r] == 5.0).all()
            continue
        err = np.abs(got[r] - want[r])
        lim = tol[r] + pu.half_step(q.dtype) * (np.abs(want[r]) + tol[r]) + pu.TINY[q.dtype]
        assert (err <= lim).all(), (r, float((err - lim).max()), float(err.max()))
        fin = np.isfinite(wl[r])
        assert np.array_equal(fin, np.isfinite(gl[r])) and (gl[r][~fin] == -np.inf).all()
        assert (np.abs(gl[r][fin] - wl[r][fin]) <= ltol[r][fin]).all()
    return out[:n]


BF, FP, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
HEADS = [(4, 2, 64), (28, 4, 128), (32, 2, 128), (8, 8, 64), (3, 1, 128), (40, 1, 64), (9, 3, 64)]
TYPES = [(BF, FP), (FP, FP), (BF, BF), (BF, E4), (FP, E4)]


@pytest.mark.parametrize("hq,hk,hd", HEADS)
@pytest.mark.parametrize("qt,cache", TYPES)
@pytest.mark.parametrize("page,layout", [(16, "hnd"), (48, "nhd")])
def test_attention_single_rows(B, hq, hk, hd, qt, cache, page, layout):
    lens = [1, 0, 2, 15, 16, 17, 47, 48, 49, 63, 64, 65, 130, 300]
    c = attn_case(lens, [1] * len(lens), hq, hk, hd, page, qt, cache, layout, hq + page, cache == E4)
    q, kc, vc, table, start, sc = c
    got = check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=1, max_len=300)
    # the same without what the caller need not know
    again = B.paged_attention(q, kc, vc, ints(table), ints(lens), k_scale=sc[0], v_scale=sc[1])
    assert torch.allclose(again.float(), got.float(), rtol=2 ** -6, atol=1e-3)


@pytest.mark.parametrize("hq,hk,hd", [(4, 2, 64), (28, 4, 128), (32, 2, 128), (5, 5, 128), (64, 1, 64)])
@pytest.mark.parametrize("qt,cache", TYPES)
@pytest.mark.parametrize("page,layout", [(32, "nhd"), (64, "hnd")])
def test_attention_blocks_of_rows(B, hq, hk, hd, qt, cache, page, layout):
    """Causal blocks, a sequence without new rows, one shorter than its rows (rows that see nothing)."""
    lens, rows = [4, 70, 129, 64, 3, 200, 5, 0, 33], [4, 3, 8, 1, 5, 2, 0, 2, 13]
    q, kc, vc, table, start, sc = attn_case(lens, rows, hq, hk, hd, page, qt, cache, layout, 7 * hq, cache == E4)
    check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=13, max_len=200)
    check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=1)  # an understated bound changes nothing


@pytest.mark.parametrize("lens,rows,hq,hk,hd,page,qt,cache", [
    ([5000], [1], 28, 4, 128, 64, BF, FP), ([9001], [4], 32, 2, 128, 16, BF, BF), ([3000, 1, 0, 2100, 17], [1, 1, 1, 3, 2], 8, 2, 64, 48, FP, FP),
    ([4097, 12], [2, 1], 16, 1, 128, 128, FP, E4), ([20011], [1], 4, 1, 64, 256, BF, FP), ([700] * 9, [3] * 9, 32, 8, 128, 16, BF, FP),
])
def test_attention_long_and_split(B, lens, rows, hq, hk, hd, page, qt, cache):
    q, kc, vc, table, start, sc = attn_case(lens, rows, hq, hk, hd, page, qt, cache, "hnd", sum(lens), cache == E4)
    check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=max(rows), max_len=max(lens))


def test_attention_large_scores(B):
    """Scores of several hundred: the running maximum carries them, late maxima rescale what was summed."""
    lens, rows = [500, 77, 4000], [1, 2, 1]
    q, kc, vc, table, start, sc = attn_case(lens, rows, 8, 2, 64, 16, BF, FP, "hnd", 5)
    check_attn(B, q * 8, kc, vc, table, lens, start, sc, scale=2.0)
    for i, n in enumerate(lens):  # keys that grow towards the end
        for p in range(n):
            kc[int(table[i, p // 16]), :, p % 16] *= p / n
    check_attn(B, q, kc, vc, table, lens, start, sc, scale=3.0)


def test_attention_not_finite_in_masked_places(B):
    """A block's later rows hold infinities and NaN: the earlier rows do not see them, the later ones do."""
    for cache, nans in ((FP, (float("inf"), float("nan"), -float("inf"))), (E4, (float("nan"),))):
        for bad in nans:
            lens, rows = [70, 35, 131], [4, 3, 20]
            q, kc, vc, table, start, sc = attn_case(lens, rows, 8, 2, 64, 16, BF, cache, "hnd", 9, cache == E4)
            clean = B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start), k_scale=sc[0], v_scale=sc[1])
            for i, (n, r) in enumerate(zip(lens, rows)):
                for p in range(n - r + 1, n):  # all but the block's first position
                    kc[int(table[i, p // 16]), :, p % 16, 5] = bad
                    vc[int(table[i, p // 16]), :, p % 16, 3] = bad
            got = B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start), k_scale=sc[0], v_scale=sc[1])
            for i in range(3):
                a = int(start[i])
                assert torch.equal(got[a], clean[a])
                assert not bool(torch.isfinite(got[a + 1:start[i + 1], :, 3].float()).any())
    # values only: what a row sees of them stays in its own dimension
    lens, rows = [40, 9], [6, 9]
    q, kc, vc, table, start, sc = attn_case(lens, rows, 4, 2, 64, 16, BF, FP, "hnd", 2)
    clean = B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start))
    for i, (n, r) in enumerate(zip(lens, rows)):
        vc[int(table[i, (n - 2) // 16]), :, (n - 2) % 16, 7] = float("inf")
    got = B.paged_attention(q, kc, vc, ints(table), ints(lens), row_start=ints(start))
    for i in range(2):
        a, b = int(start[i]), int(start[i + 1])
        assert torch.equal(got[a:b - 2], clean[a:b - 2])
        assert bool((got[b - 2:b, :, 7] == float("inf")).all())
        rest = [d for d in range(64) if d != 7]
        assert torch.equal(got[b - 2:b][:, :, rest], clean[b - 2:b][:, :, rest])


def test_attention_pages_that_do_not_exist(B):
    """Page ids outside the pool are left out; a sequence of only such pages gives zeros; a length beyond the table ends there."""
    lens, rows = [100, 50, 64], [2, 1, 1]
    q, kc, vc, table, start, sc = attn_case(lens, rows, 8, 2, 128, 16, BF, FP, "nhd", 4)
    table[0, 2], table[0, 6], table[1, :] = -1, kc.shape[0], 2 ** 30
    check_attn(B, q, kc, vc, table, lens, start, sc)
    table = table[:, :4].copy()
    check_attn(B, q, kc, vc, table, [1000, 50, 2 ** 31 - 1], start, sc)
    got = B.paged_attention(q[:1], kc, vc, ints(table[2:]), ints([-5]))
    assert float(got.abs().max()) == 0.0


def test_attention_bad_row_starts_stay_inside(B):
    """Row starts that leave the rows or run backwards read and write nothing outside."""
    q, kc, vc, table, start, sc = attn_case([30, 40, 50], [1, 1, 1], 4, 2, 64, 16, BF, FP, "hnd", 6)
    out = torch.full((9, 4, 64), 5.0, dtype=BF, device="cuda")
    B.paged_attention(q, kc, vc, ints(table), ints([30, 40, 50]), row_start=ints([-3, 1, 0, 7]), out=out[3:6])
    torch.cuda.synchronize()
    assert bool((out[:3] == 5.0).all()) and bool((out[6:] == 5.0).all())


@pytest.mark.parametrize("max_rows,max_len", [(1, 1), (1, 128), (2, 300), (64, 100000), (0, 0), (8, 129)])
def test_attention_hints_change_no_result(B, max_rows, max_len):
    """What the caller knows of rows and lengths, understated (segments are then not cut, or tiles come in several blocks) or
    overstated."""
    lens, rows = [300, 5, 2000, 128, 129], [3, 1, 9, 2, 1]
    q, kc, vc, table, start, sc = attn_case(lens, rows, 14, 2, 64, 16, BF, FP, "hnd", 21)
    check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=max_rows, max_len=max_len)


def test_attention_many_sequences(B):
    """More sequences than a CTA has threads, most of them short, some without rows."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 40, 700)]
    rows = [int(x) for x in rng.integers(0, 3, 700)]
    lens[13], lens[600], rows[13], rows[600] = 900, 1500, 1, 2
    q, kc, vc, table, start, sc = attn_case(lens, rows, 4, 2, 64, 16, BF, FP, "nhd", 22)
    check_attn(B, q, kc, vc, table, lens, start, sc, max_rows=2, max_len=1500)


def test_attention_strides(B):
    """Queries and outputs as slices of wider rows, heads apart, any element as the first."""
    lens = [33, 100]
    q, kc, vc, table, start, sc = attn_case(lens, [1, 1], 6, 3, 64, 16, BF, FP, "hnd", 8)
    want = B.paged_attention(q, kc, vc, ints(table), ints(lens))
    for off, pad in ((1, 3), (8, 64), (2, 2)):
        wide_q = torch.full((2, 7, 64 + pad), 9.0, dtype=BF, device="cuda").view(-1)
        qv = wide_q[off:].as_strided((2, 6, 64), (7 * (64 + pad), 64 + pad, 1), off)
        qv.copy_(q)
        wide_o = torch.full_like(wide_q, 7.0)
        ov = wide_o.as_strided((2, 6, 64), (7 * (64 + pad), 64 + pad, 1), off)
        B.paged_attention(qv, kc, vc, ints(table), ints(lens), out=ov)
        assert torch.equal(ov, want)
        ov.fill_(7.0)
        assert bool((wide_o == 7.0).all())


def test_attention_beyond_4_gib(B):
    pages, page = 33000, 16
    kc, vc = (torch.zeros((pages, 64, page, 128), dtype=E4, device="cuda") for _ in "kv")
    vc[-1, :, 3], vc[0, :, 2] = 2.0, 4.0
    q = torch.ones((1, 64, 128), dtype=BF, device="cuda")
    got = B.paged_attention(q, kc, vc, ints([[pages - 1, 0]]), ints([32]))
    assert bool((got == 6.0 / 32).all())


# ------------------------------------------------------------------ sampling
def run_sample(B, z, u, T=None, k=None, p=None, m=None, lo=None, hi=None):
    f = lambda v: None if v is None else torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    n = z.shape[0]
    lp = torch.full((n,), 9.0, device="cuda")
    t = B.sample(z, f(u), temperature=f(T), top_k=None if k is None else ints(k), top_p=f(p), min_p=f(m),
                 id_lo=None if lo is None else ints(lo), id_hi=None if hi is None else ints(hi), logprob=lp)
    zz = z.double().cpu().numpy()
    f32 = lambda v, d: np.full(n, d) if v is None else np.asarray(v, np.float32).astype(np.float64)  # noqa: E731
    T, p, m, u = f32(T, 1.0), f32(p, 1.0), f32(m, 0.0), f32(u, 0.0)
    k = [0] * n if k is None else k
    lo, hi = [0] * n if lo is None else lo, [z.shape[1]] * n if hi is None else hi
    want = [pu.sample(zz[i], lo[i], hi[i], T[i], k[i], p[i], m[i], u[i]) for i in range(n)]
    assert t.tolist() == [w[0] for w in want]
    for g, (_, w) in zip(lp.tolist(), want):
        # 64-bit arithmetic, rounded once
        assert g == w or abs(g - w) <= 2.0 ** -24 * abs(w) + 1e-9
    return t


@pytest.mark.parametrize("V", [1, 2, 31, 33, 511, 1024, 6561, 16384, 16385, 50001, 151936])
@pytest.mark.parametrize("dtype", [torch.float32, BF, FP])
@pytest.mark.parametrize("scale", [0.0, 0.3, 3.0, 30.0])
def test_sample(B, V, dtype, scale):
    n = 10
    gen = torch.Generator("cuda").manual_seed(V)
    z = (torch.randn((n, V + 3), generator=gen, device="cuda") * scale).to(dtype)[:, :V]
    u = torch.rand(n, generator=gen, device="cuda").clamp(max=1 - 2.0 ** -24).tolist()
    T, k = [1.0, 0.7, 0.0, 2.5, 0.05, 1.0, 0.9, 1.0, 1e-6, 1.0], [0, 50, 0, 1, 3, 100000, 0, V, 0, 4000]
    p, m = [0.9, 1.0, 0.5, 0.99, 1.0, 1e-9, 0.3, 0.999, 0.9, 0.95], [0.0, 0.0, 0.0, 0.0, 0.1, 0.0, 0.02, 0.5, 0.0, 1e-4]
    run_sample(B, z, u, T, k, p, m)
    run_sample(B, z, u)
    lo = [0, V // 2, 0, V // 3, V - 1, -5, 0, 1, 0, V]
    hi = [V, V, V // 2 + 1, V, V, V + 9, 1, V, V // 7, V]
    run_sample(B, z, u, T, k, p, m, lo, hi)


@pytest.mark.parametrize("V", [100, 20000, 151936])
@pytest.mark.parametrize("dtype", [torch.float32, BF])
@pytest.mark.parametrize("shift", [0.0, -500.0, 3000.0])
def test_sample_light_logits(B, V, dtype, shift):
    """min-p whose border lies near zero, far from it, behind every id, or before the second one; after cuts that are
    tighter, and after a bin that had to be divided."""
    n = 12
    gen = torch.Generator("cuda").manual_seed(V + 1)
    z = torch.randn((n, V), generator=gen, device="cuda") * 2.0
    z -= z.max(1, keepdim=True).values  # (the border at ln(min_p) T is around zero in the rows that are raised by it)
    m = [1e-30, 1e-6, 0.01, 0.3, 1 - 2.0 ** -24, 1.0, 0.05, 0.05, 1e-3, 1e-3, 0.2, 1e-12]
    T = [1.0, 0.5, 1.0, 2.0, 1.0, 1.0, 1.0, 1.0, 0.7, 3.0, 1.0, 1.0]
    for i in (1, 2, 3, 9):
        z[i] -= T[i] * float(np.log(m[i]))
    z = z + shift
    z[11, V // 3:] = z[11, 0]  # so many equal that their bin is divided, or is one number
    z = z.to(dtype)
    u = torch.rand(n, generator=gen, device="cuda").clamp(max=1 - 2.0 ** -24).tolist()
    run_sample(B, z, u, T, None, None, m)
    run_sample(B, z, u, T, [0, 0, 0, 0, 0, 0, 5, 0, 0, 70, 0, V // 2], [1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 0.5, 0.9, 0.9, 0.05, 0.9], m)


def test_sample_by_hand(B):
    """Weights that are powers of two, so that every border is exact: the first id beyond u times the kept mass."""
    z = torch.tensor([[-2.0, 0.0, -2.0, -1.0]], device="cuda").expand(8, 4).contiguous() * 0.693147180559945
    run_sample(B, z, [0.0, 0.4, 0.6, 0.7, 0.8, 0.9, 0.99, 0.3])
    flat = torch.zeros((8, 8), device="cuda")
    for dtype in (torch.float32, BF, FP):
        zz = flat.to(dtype)
        u = [0.0, 0.124, 0.125, 0.5, 0.874, 0.875, 0.9999, 0.25]
        assert run_sample(B, zz, u).tolist() == [0, 0, 1, 4, 6, 7, 7, 2]
        assert run_sample(B, zz, u, k=[4] * 8).tolist() == [0, 0, 0, 2, 3, 3, 3, 1]
        assert run_sample(B, zz, u, p=[0.5] * 8).tolist() == [0, 0, 0, 2, 3, 3, 3, 1]
        assert run_sample(B, zz, u, k=[4] * 8, p=[0.5] * 8).tolist() == [0, 0, 0, 1, 1, 1, 1, 0]
        assert run_sample(B, zz, u, m=[1.0] * 8, lo=[2] * 8).tolist()[0] == 2
    # the two zeros are one number, numbers too small for fp32's normal range are not zero
    z = torch.tensor([[0.0, -0.0, 0.0, -0.0], [-0.0, 1e-40, 0.0, -1e-40]], device="cuda")
    assert run_sample(B, z, [0.3, 0.1]).tolist() == [1, 1]
    assert run_sample(B, z, [0.3, 0.1], T=[0.0, 0.0]).tolist() == [0, 1]


@pytest.mark.parametrize("V", [40, 30000, 151936])
def test_sample_masks(B, V):
    """Ids ruled out by minus infinity, by NaN, by the type's lowest value; rows without any id; infinite logits."""
    inf = float("inf")
    z = torch.randn((9, V), generator=torch.Generator("cuda").manual_seed(V), device="cuda")
    z[0, ::2] = -inf
    z[1, 1:] = -inf
    z[2, 3:] = float("nan")
    z[3] = -inf
    z[4] = float("nan")
    z[5, ::3] = torch.finfo(torch.float32).min
    z[6] = torch.finfo(torch.float32).min
    z[7, 5], z[7, 9] = inf, inf
    z[8, 4] = 3e38
    u = [0.7, 0.2, 0.9, 0.5, 0.5, 0.999, 0.35, 0.6, 0.1]
    got = run_sample(B, z, u, T=[0.8] * 9, p=[0.95] * 9).tolist()
    assert got[3] == got[4] == -1 and got[7] == 9 and got[8] == 4
    run_sample(B, z, u)
    run_sample(B, z, u, T=[0.0] * 9)
    run_sample(B, z, u, k=[2] * 9, m=[0.3] * 9)


def test_sample_settings_out_of_range(B):
    """Settings lie on the device and cannot be refused: each odd value means what the header says."""
    nan, inf = float("nan"), float("inf")
    z = torch.randn((8, 300), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    best = z.argmax(1).tolist()
    u = torch.tensor([0.5] * 8, device="cuda")
    f = lambda v: torch.tensor(v, device="cuda")  # noqa: E731
    T = f([0.0, -1.0, nan, 1e-38, 1.0, 1.0, 1.0, 1.0])
    p = f([1.0, 1.0, 1.0, 1.0, 0.0, -2.0, 1.0, 1.0])
    m = f([0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1.0, 7.0])
    assert B.sample(z, u, temperature=T, top_p=p, min_p=m).tolist() == best
    want = B.sample(z, u)
    assert torch.equal(B.sample(z, u, top_k=ints([-3, 0, 300, 301, 2 ** 31 - 1, -2 ** 31, 0, 0]), top_p=f([nan, 1.0, 9.0, inf] * 2),
                                min_p=f([nan, -1.0, 0.0, -inf] * 2)), want)
    first = B.sample(z, f([0.0] * 8))
    assert torch.equal(B.sample(z, f([nan, -1.0, -inf, 0.0] * 2)), first)
    # id ranges: cut to the row, empty where they run backwards
    lo, hi = ints([-2 ** 31, 5, 300, 2 ** 31 - 1, 0, 7, 0, 299]), ints([2 ** 31 - 1, -2 ** 31, 301, 2 ** 31 - 1, 0, 3, 300, 2 ** 31 - 1])
    got = B.sample(z, u, id_lo=lo, id_hi=hi)
    assert got[[0, 6]].tolist() == want[[0, 6]].tolist() and got[1:6].tolist() == [-1] * 5 and int(got[7]) == 299
    flat = torch.zeros((2, 300), device="cuda")
    assert B.sample(flat, f([1.0, 5.0])).tolist() == [299, 299]
    assert B.sample(flat, f([0.5, 0.5]), temperature=f([inf, inf])).tolist() == [150, 150]


@pytest.mark.parametrize("V,kind", [(151936, "equal"), (151936, "two"), (262144, "steps"), (6000, "equal"), (100000, "near"), (40000, "bf16")])
def test_sample_many_equal_logits(B, V, kind):
    """Rows whose border lies among thousands of equal or nearly equal logits."""
    gen = torch.Generator("cuda").manual_seed(V)
    n = 6
    z = torch.randn((n, V), generator=gen, device="cuda")
    if kind == "equal":
        z[:] = -3.5
    elif kind == "two":
        z = (z > 0).float()
    elif kind == "steps":
        z = (z * 4).round() / 4
    elif kind == "near":  # neighbours in the last bits
        z = 1.0 + torch.randint(0, 5000, (n, V), generator=gen, device="cuda") * 2.0 ** -23
    else:
        z = z.to(BF)
    u = torch.rand(n, generator=gen, device="cuda").tolist()
    run_sample(B, z, u)
    run_sample(B, z, u, p=[0.9, 0.5, 0.3, 0.1, 0.999, 0.7], k=[0, 0, V // 2, 77, 5000, 1])


# ------------------------------------------------------------------ how the calls are made
def test_another_stream_and_a_captured_step(B):
    """All four calls in one graph, replayed while lengths, tables, rows and settings change underneath, and on a side stream."""
    hq, hk, hd, page, n_seqs, V = 8, 2, 64, 16, 3, 5000
    gen = torch.Generator("cuda").manual_seed(1)
    pages = 40
    kc, vc = (torch.zeros((pages, hk, page, hd), dtype=FP, device="cuda") for _ in "kv")
    table, ring = torch.full((n_seqs, 8), -1, dtype=torch.int32, device="cuda"), torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    lens, rows, queue = ints([0, 0, 0]), ints([0, 0, 0]), ints([0, pages])
    rope = torch.randn((128, hd // 2, 2), generator=gen, device="cuda")
    most = 24
    x = torch.zeros((most, hq + 2 * hk, hd), dtype=BF, device="cuda")
    z, u = torch.zeros((n_seqs, V), device="cuda"), torch.zeros(n_seqs, device="cuda")

    def step():
        m = B.page_map(lens, rows, table, ring, queue, page, max_rows=most)
        q = B.paged_append(x[:, hq:hq + hk], x[:, hq + hk:], kc, vc, m.slot_map, q=x[:, :hq], row_pos=m.row_pos, rope=rope)
        o = B.paged_attention(q, kc, vc, table, m.seq_len, row_start=m.row_start)
        t = B.sample(z, u, top_p=torch.full_like(u, 0.9))
        return m, q, o, t

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m, q, o, t = step()
    at, host_len, host_q = ring.clone(), [0, 0, 0], [0, pages]
    for turn, add in enumerate([[5, 16, 1], [1, 1, 1], [3, 0, 17], [1, -1, 1], [2, 20, 1]]):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        z.copy_(torch.randn(z.shape, generator=gen, device="cuda"))
        u.copy_(torch.rand(u.shape, generator=gen, device="cuda"))
        rows.copy_(ints(add))
        ref = pu.page_map(host_len, add, table.cpu().numpy(), ring.cpu().numpy(), host_q, page, most)
        graph.replay()
        assert int(m.status) == 0 and np.array_equal(m.slot_map.cpu().numpy(), ref[7]) and np.array_equal(table.cpu().numpy(), ref[0])
        dbl = lambda a: a.double().cpu().numpy()  # noqa: E731
        want, _, tol, _ = pu.attend(dbl(q), dbl(kc), dbl(vc), ref[0], ref[2], ref[4], hd ** -0.5, 2.0 ** -11)
        got = dbl(o)
        for r in range(int(ref[4][-1])):
            assert (np.abs(got[r] - want[r]) <= tol[r] + pu.half_step(BF) * (np.abs(want[r]) + tol[r])).all()
        assert t.tolist() == [pu.sample(dbl(z)[i], 0, V, 1.0, 0, float(np.float32(0.9)), 0.0, float(u[i]))[0] for i in range(n_seqs)]
        host_len, host_q = [int(v) for v in ref[2]], [int(v) for v in ref[3]]
        lens.copy_(m.seq_len)
        queue.copy_(m.queue)
    assert torch.equal(at.sort().values, torch.arange(pages, device="cuda", dtype=torch.int32))


def test_calls_that_overlap(B):
    """The same attention on several streams at once, each with scratch of its own: every one gets the same result."""
    lens = [3000, 200, 999]
    q, kc, vc, table, start, sc = attn_case(lens, [1] * 3, 28, 4, 128, 16, BF, FP, "hnd", 12)
    t, n = ints(table), ints(lens)
    want = B.paged_attention(q, kc, vc, t, n)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(4)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(B.paged_attention(q, kc, vc, t, n))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_binding_refuses_and_leaves_outputs_alone(B):
    """What the binding checks before the ABI sees it: types, sizes, layouts and numbers that do not fit."""
    lens, page, hd = [20, 5], 16, 64
    q, kc, vc, table, start, sc = attn_case(lens, [1, 1], 4, 2, hd, page, FP, FP, "hnd", 3)
    t, n = ints(table), ints(lens)
    out = torch.full_like(q, 7.0)
    z, u, token = torch.zeros((2, 9), device="cuda"), torch.zeros(2, device="cuda"), ints([-5, -5])
    k, slots = torch.zeros((2, 2, hd), dtype=FP, device="cuda"), ints([0, 1], torch.int64)
    rope = torch.zeros((32, hd // 2, 2), device="cuda")
    i = ints([1, 1])
    big = ints(np.zeros((2, 4)))
    attend = lambda *a, **kw: B.paged_attention(*a, out=out, **kw)  # noqa: E731
    draw = lambda *a, **kw: B.sample(*a, token=token, **kw)  # noqa: E731
    before = kc.view(torch.int16).clone()  # (bits: unused places hold NaN)
    calls = [lambda: attend(q, kc, vc, t, n, max_len=2 ** 31), lambda: attend(q, kc, vc, t, n, max_rows="1"),
             lambda: attend(q, kc, vc, t, n, scale="x"), lambda: attend(q, kc, vc, t.long(), n), lambda: attend(q, kc, vc, t[:1], n),
             lambda: attend(q, kc, vc, t, n.long()), lambda: attend(q, kc, vc.float(), t, n), lambda: attend(q, kc, vc, t, n, row_start=n),
             lambda: attend(q[..., :32], kc, vc, t, n), lambda: attend(q.to(BF), kc, vc, t, n), lambda: attend(q, kc, vc, t, n.cpu()),
             lambda: attend(q, kc, vc, t, n, lse=u), lambda: attend(q, kc, vc, t, n, scratch=torch.zeros(16, dtype=torch.uint8, device="cuda")),
             lambda: draw(z, u.double()), lambda: draw(z, u[:1]), lambda: draw(z.double(), u), lambda: draw(z.t(), u),
             lambda: draw(z, u, top_k=u), lambda: draw(z, u, temperature=i), lambda: draw(z, u, logprob=u.cpu()),
             lambda: B.paged_append(k, k, kc, vc, slots.int()), lambda: B.paged_append(k, k.float(), kc, vc, slots),
             lambda: B.paged_append(k[:, :1], k, kc, vc, slots), lambda: B.paged_append(k, k, kc, vc, slots, rope=rope),
             lambda: B.paged_append(k, k, kc, vc, slots, q=k.float()), lambda: B.paged_append(k, k, kc, vc, slots, k_scale=u[:1]),
             lambda: B.page_map(i, i, big, ints(range(8)), ints([0, 8]), 2 ** 31, max_rows=4),
             lambda: B.page_map(i, i[:1], big, ints(range(8)), ints([0, 8]), 16, max_rows=4),
             lambda: B.page_map(i, i, big, ints(range(8)), ints([0, 8, 1]).long(), 16, max_rows=4)]
    for f in calls:
        with pytest.raises(B.SparskError) as e:
            f()
        assert e.value.code == B.EINVAL
    torch.cuda.synchronize()
    assert (out == 7).all() and (token == -5).all() and torch.equal(kc.view(torch.int16), before)


def test_threads_with_streams_of_their_own(B):
    """The binding lets go of Python's lock while it launches: calls of several threads stay apart."""
    from concurrent.futures import ThreadPoolExecutor
    lens = [700, 33, 1]
    q, kc, vc, table, start, sc = attn_case(lens, [1] * 3, 8, 2, 128, 16, BF, FP, "nhd", 21)
    t, n = ints(table), ints(lens)
    z, u = torch.randn((3, 5000), device="cuda"), torch.rand(3, device="cuda")
    want, tokens = B.paged_attention(q, kc, vc, t, n), B.sample(z, u)
    torch.cuda.synchronize()

    def work(_):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got = [(B.paged_attention(q, kc, vc, t, n), B.sample(z, u)) for _ in range(40)]
        s.synchronize()
        return all(torch.equal(a, want) and torch.equal(b, tokens) for a, b in got)

    with ThreadPoolExecutor(4) as pool:
        assert all(pool.map(work, range(4)))
