"""What the operators of a paged serving step are timed on, and their plain forms.

A serving program that shares one pool of cache pages between its requests makes four calls around
the model's products, in this order:
  page_map         from the requests' lengths: pages for what is new, the table of every request's
                   pages, and where each new row goes
  paged_append     new queries and keys turned to their positions, keys and values put into the pages
  paged_attention  the new rows over their requests' pages
  sample           a token a request, by its own temperature, top-k, top-p and min-p
`own` says whether a pass makes the library's calls or computes the same in elementary torch
operations, in 32 bits (the sampling in 64: a draw is decided at the border between two ids).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "e4m3": 1}
LARGEST = {"bf16": None, "fp16": 65504.0, "e4m3": 448.0}


# ------------------------------------------------------------------ cases
def _attend(name, seqs, len_lo, len_hi, heads, page, rows=1, q="bf16", cache="fp16", layout="hnd"):
    return dict(name=name, kind="attend", seqs=seqs, len_lo=len_lo, len_hi=len_hi, q_heads=heads[0], kv_heads=heads[1],
                head_dim=heads[2], page=page, rows=rows, q=q, cache=cache, layout=layout)


def _append(name, rows, heads, page, x="bf16", cache="fp16", layout="hnd", pad=0):
    return dict(name=name, kind="append", rows=rows, q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2], page=page, x=x,
                cache=cache, layout=layout, pad=pad)


def _map(name, seqs, len_lo, len_hi, page, prompts, gone):
    return dict(name=name, kind="map", seqs=seqs, len_lo=len_lo, len_hi=len_hi, page=page, prompts=prompts, gone=gone)


def _sample(name, rows, text, speech, scale, x="fp32", mixed=True):
    return dict(name=name, kind="sample", rows=rows, text=text, speech=speech, scale=scale, x=x, mixed=mixed)


def listed():
    return [
        # a decode step of a loaded server: 64 requests, one new row each, every now and then a new page
        _map("map_b64", 64, 256, 2048, 16, 0, 0),
        # requests come and go: a few hundred in flight, 24 new prompts among them, 16 that have ended
        _map("map_prompts_b300", 300, 100, 8192, 32, 24, 16),
        # the keys and values of one decode step's 64 rows, and their queries
        _append("append_b64", 64, (28, 4, 128), 16),
        # a chunk of prompts, of which the last rows are padding, into pages of 8-bit numbers
        _append("append_prompt_e4m3", 4001, (32, 2, 128), 64, cache="e4m3", layout="nhd", pad=95),
        # the smallest call: the four-layer model's heads, one request, a short prompt
        _attend("attend_tiny_b1", 1, 32, 32, (4, 2, 64), 16),
        # one listener after a long conversation: all of the GPU on one sequence
        _attend("attend_b1_8k", 1, 8191, 8191, (28, 4, 128), 64),
        # a loaded server: 64 requests of ragged length on small pages
        _attend("attend_b64_ragged", 64, 256, 2048, (28, 4, 128), 16),
        # long conversations of the 40-layer backbone's heads, a cache in bf16
        _attend("attend_b64_long_bf16", 64, 8192, 8192, (32, 2, 128), 64, cache="bf16"),
        # refresh steps: one to four rows a request, pages of 8-bit numbers, heads side by side in a position
        _attend("attend_refresh_e4m3", 48, 700, 4000, (32, 2, 128), 32, rows=4, cache="e4m3", layout="nhd"),
        # a speech token of one listener
        _sample("sample_speech_b1", 1, 0, 6561, 1.2, mixed=False),
        # a text token of each of 16 requests with settings of their own, from 16-bit logits
        _sample("sample_text_b16_bf16", 16, 151552, 0, 2.0, x="bf16"),
        # a loaded server whose requests are at text or at speech, nearly flat predictions
        _sample("sample_mixed_b64", 64, 151936, 6561, 0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(4, 2, 64), (28, 4, 128), (32, 2, 128), (32, 8, 128), (8, 8, 64), (16, 1, 128)]


def draw(rng):
    kind = rng.choice(["attend"] * 5 + ["sample"] * 3 + ["append"] * 2 + ["map"] * 2)
    layout, page = rng.choice(["hnd", "nhd"]), rng.choice([16, 16, 32, 48, 64, 128])
    cache = rng.choice(["fp16", "fp16", "bf16", "e4m3"])
    if kind == "attend":
        heads = rng.choice(HEADS)
        seqs = _log(rng, 1, 128)
        hi = _log(rng, 20, min(32768, 1000000 // (seqs * heads[1]) * 128 // heads[2]))
        q = "bf16" if cache == "bf16" else rng.choice(["bf16", "bf16", "fp16"])
        c = _attend("", seqs, _log(rng, 1, hi), hi, heads, page, rng.choice([1, 1, 1, 2, 3, 4, 8]), q, cache, layout)
    elif kind == "append":
        rows = _log(rng, 1, 8000)
        c = _append("", rows, rng.choice(HEADS), page, rng.choice(["bf16", "bf16", "fp16", "fp32"]), cache, layout,
                    rng.choice([0, 0, rows // 7]))
    elif kind == "map":
        seqs = _log(rng, 1, 1000)
        hi = _log(rng, 20, 8192)
        c = _map("", seqs, _log(rng, 1, hi), hi, page, rng.choice([0, seqs // 10, seqs // 3]), rng.choice([0, seqs // 12]))
    else:
        text = _log(rng, 30, 160000)
        c = _sample("", _log(rng, 1, 64), text, rng.choice([0, 0, 1, text // 9, 6561]), rng.choice([0.3, 1.0, 2.0, 4.0]),
                    rng.choice(["fp32", "fp32", "bf16", "fp16"]), rng.random() < 0.8)
    del c["name"]
    return c


def _spread(n, lo, hi):
    """n lengths, evenly over [lo, hi] and shuffled."""
    out = [lo + (hi - lo) * i // max(1, n - 1) if n > 1 else hi for i in range(n)]
    random.Random(n).shuffle(out)
    return out


def _rows_of(case):
    """New rows of every sequence of an attention case: every third one a block of the most it may be."""
    lens = _spread(case["seqs"], case["len_lo"], case["len_hi"])
    return lens, [min(n, case["rows"] if i % 3 == 0 else 1 + i % case["rows"]) for i, n in enumerate(lens)]


def _steps_of(case):
    """(length, rows) of every sequence of a page map: prompts begin at nothing, -1 is a sequence that has ended."""
    lens = _spread(case["seqs"], case["len_lo"], case["len_hi"])
    rows = [1] * len(lens)
    for i in range(case["prompts"]):
        at = (i * 7 + 3) % len(lens)
        rows[at], lens[at] = max(1, lens[at] // 3), 0
    for i in range(case["gone"]):
        at = (i * 11 + 5) % len(lens)
        rows[at] = -1
    return lens, rows


# ------------------------------------------------------------------ inputs
def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _randn(gen, *shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)


def _pool(gen, case, pages):
    """A page pool as [page][head][position][dim], however it lies in memory; 8-bit ones hold numbers with a scale a head."""
    h, p, d = case["kv_heads"], case["page"], case["head_dim"]
    x = _randn(gen, *((pages, h, p, d) if case["layout"] == "hnd" else (pages, p, h, d)), dtype=torch.float16)
    if case["cache"] == "e4m3":
        x = (x * 16).clamp_(-448, 448)
    x = x.to(DTYPES[case["cache"]])
    return x if case["layout"] == "hnd" else x.transpose(1, 2)


def _scales(gen, case):
    if case["cache"] != "e4m3":
        return None
    return torch.rand(case["kv_heads"], device="cuda", generator=gen) * 0.02 + 1 / 16


def _prepare_attend(case, gen):
    lens, rows = _rows_of(case)
    n, blocks = sum(rows), [-(-x // case["page"]) for x in lens]
    pages = sum(blocks) + 7
    perm = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(blocks) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = perm[at:at + b]
        at += b
    start = [sum(rows[:i]) for i in range(len(rows) + 1)]
    seq_of = [i for i, r in enumerate(rows) for _ in range(r)]
    pos = [lens[i] - r + j for i, r in enumerate(rows) for j in range(r)]
    q = _randn(gen, n, case["q_heads"], case["head_dim"]).to(DTYPES[case["q"]])
    return dict(case=case, q=q, k=_pool(gen, case, pages), v=_pool(gen, case, pages), table=table, lens=_ints(lens),
                row_start=_ints(start), row_seq=_ints(seq_of), row_pos=_ints(pos), max_len=max(lens), max_rows=max(rows),
                k_scale=_scales(gen, case), v_scale=_scales(gen, case), out=torch.zeros_like(q))


def _rope_table(positions, head_dim):
    half = head_dim // 2
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None]
    a = a * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _prepare_append(case, gen):
    n, hq, hk, d = case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    pages = -(-n // case["page"]) * 2 + 3
    x = _randn(gen, n, hq + 2 * hk, d).to(DTYPES[case["x"]])  # a row of the products: queries, keys, values
    slots = torch.randperm(pages * case["page"], device="cuda", generator=gen)[:n]
    pos = torch.randint(0, 8192, (n,), device="cuda", generator=gen).to(torch.int32)
    if case["pad"]:
        slots[n - case["pad"]:] = -1
    out = torch.float16 if case["x"] == "fp16" else torch.bfloat16
    return dict(case=case, q=x[:, :hq], k=x[:, hq:hq + hk], v=x[:, hq + hk:], slots=slots, pos=pos, rope=_rope_table(8192, d),
                k_cache=_pool(gen, case, pages), v_cache=_pool(gen, case, pages), k_scale=_scales(gen, case),
                v_scale=_scales(gen, case), q_out=torch.zeros((n, hq, d), dtype=out, device="cuda"))


def _prepare_map(case, gen):
    lens, rows = _steps_of(case)
    P = case["page"]
    blocks = [-(-x // P) for x in lens]
    after = [-(-(x + max(r, 0)) // P) for x, r in zip(lens, rows)]
    need = sum(max(0, b - a) for a, b in zip(blocks, after))
    pages = sum(blocks) + need + 37
    perm = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(max(after), max(blocks)) + 2), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = perm[at:at + b]
        at += b
    # the queue of free pages lies anywhere in its ring
    head, free = int(torch.randint(0, pages, (1,), device="cuda", generator=gen)), pages - at
    ring = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free, device="cuda")) % pages] = perm[at:]
    total = sum(max(r, 0) for r in rows)
    most = -(-total // 64) * 64  # a program's buffers hold a round number of rows
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(case=case, lens=_ints(lens), rows=_ints(rows), table=table, ring=ring, queue=_ints([head, free]), most=most,
                out=dict(seq_len=i32(len(lens)), queue=i32(2), row_start=i32(len(lens) + 1), row_seq=i32(most), row_pos=i32(most),
                         slot_map=torch.zeros(most, dtype=torch.int64, device="cuda"), status=i32(1)))


def _prepare_sample(case, gen):
    n, V = case["rows"], case["text"] + case["speech"]
    z = (_randn(gen, n, V) * case["scale"]).to(DTYPES[case["x"]])
    u = torch.rand(n, device="cuda", generator=gen).clamp_(max=1 - 2.0 ** -24)
    text = [case["text"] > 0 and (case["speech"] == 0 or i % 3 > 0) for i in range(n)]
    lo, hi = _ints([0 if t else case["text"] for t in text]), _ints([case["text"] if t else V for t in text])
    pick = lambda v: [v[(i * 5 + i // 3) % len(v)] if case["mixed"] else v[0] for i in range(n)]  # noqa: E731
    f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    if case["mixed"]:  # ids that a request has ruled out, never all of them
        z[::4, ::5] = -math.inf
        z.scatter_(1, lo.long()[:, None], 0.0)
    return dict(case=case, z=z, u=u, lo=lo, hi=hi, temperature=f32(pick([0.7, 1.0, 0.0, 0.85, 1.3])),
                top_k=_ints(pick([0, 50, 0, 20, 1000, 0, 1])), top_p=f32(pick([0.9, 1.0, 0.95, 0.5])),
                min_p=f32(pick([0.0, 0.0, 0.05, 0.0, 0.2])), token=_ints([0] * n), logprob=f32([0.0] * n))


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    return {"attend": _prepare_attend, "append": _prepare_append, "map": _prepare_map, "sample": _prepare_sample}[case["kind"]](case, gen)


# ------------------------------------------------------------------ plain forms
def _plain_attend(s):
    c, table = s["case"], s["table"].long()
    hk, d, g, P = c["kv_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"], c["page"]
    at = torch.arange(s["max_len"], device="cuda")
    pages = table[:, at // P].clamp(min=0)  # [seqs, positions]
    k, v = (x[pages, :, at % P].float().transpose(1, 2) for x in (s["k"], s["v"]))  # [seqs, heads, positions, dim]
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"][:, None, None], v * s["v_scale"][:, None, None]
    R, n = s["max_rows"], s["q"].shape[0]
    seq, place = s["row_seq"].long(), torch.arange(n, device="cuda") - s["row_start"].long()[s["row_seq"].long()]
    q = torch.zeros((len(table), R, hk, g, d), device="cuda")
    q[seq, place] = s["q"].float().view(n, hk, g, d)
    scores = q.permute(0, 2, 1, 3, 4).reshape(-1, hk, R * g, d) @ k.transpose(2, 3) / math.sqrt(d)
    last = torch.full((len(table), R), -1, device="cuda")
    last[seq, place] = s["row_pos"].long()
    seen = at <= last[:, :, None]
    seen = seen[:, None, :, None].expand(-1, hk, R, g, -1).reshape(scores.shape)
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    w = torch.exp(scores - top)
    o = (w @ v) / w.sum(-1, keepdim=True)
    o = o.view(-1, hk, R, g, d).permute(0, 2, 1, 3, 4)[seq, place]
    return o.reshape(s["q"].shape).to(s["q"].dtype)


def _turn(x, cs):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)


def _hold(x, scale, cache):
    x = x if scale is None else x / scale[:, None]
    return (x if LARGEST[cache] is None else x.clamp(-LARGEST[cache], LARGEST[cache])).to(DTYPES[cache])


def _plain_append(s):
    c, cs = s["case"], s["rope"][s["pos"].long()][:, None]
    q = _turn(s["q"].float(), cs).to(s["q_out"].dtype)
    keep = (s["slots"] >= 0)[:, None, None]
    page = torch.where(s["slots"] >= 0, s["slots"], s["slots"][0])  # a row that is left out writes the first row once more
    page, at = page // c["page"], page % c["page"]
    for x, scale, cache in ((_turn(s["k"].float(), cs), s["k_scale"], s["k_cache"]), (s["v"].float(), s["v_scale"], s["v_cache"])):
        cache[page, :, at] = _hold(torch.where(keep, x, x[:1]), scale, c["cache"])
    return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_map(s):
    P, ring, most = s["case"]["page"], s["ring"], s["most"]
    lens, rows, table = s["lens"].long(), s["rows"].long(), s["table"]
    head, free, cap, room = s["queue"][0].long(), s["queue"][1].long(), len(ring), table.shape[1]
    gone, more = rows < 0, rows.clamp(min=0)
    had = (lens + P - 1) // P
    after = torch.where(gone, 0, lens + more)
    has = (after + P - 1) // P
    grow, back = torch.where(gone, 0, has - had), torch.where(gone, had, 0)
    start = torch.cat([more.new_zeros(1), more.cumsum(0)])
    ok = (grow.sum() <= free) & (has <= room).all() & (start[-1] <= most) & (free + back.sum() <= cap)
    j = torch.arange(room, device="cuda")
    taken = ring[(head + (grow.cumsum(0) - grow)[:, None] + j - had[:, None]) % cap]
    table.copy_(torch.where(ok & (j >= had[:, None]) & (j < has[:, None]), taken, table))
    put = torch.where(ok & (j < back[:, None]), (head + free + (back.cumsum(0) - back)[:, None] + j) % cap, cap)
    ring.copy_(torch.cat([ring, ring[:1]]).scatter(0, put.view(-1), table.view(-1))[:cap])
    r = torch.arange(most, device="cuda")
    seq = torch.searchsorted(start[1:], r, right=True).clamp(max=len(lens) - 1)
    pos = lens[seq] + r - start[seq]
    live = ok & (r < start[-1])
    slot = table[seq, (pos // P).clamp(max=room - 1)].long() * P + pos % P
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(table=table, ring=ring, seq_len=i32(torch.where(ok, after, lens)),
                queue=i32(torch.stack([torch.where(ok, (head + grow.sum()) % cap, head), torch.where(ok, free - grow.sum() + back.sum(), free)])),
                row_start=i32(torch.where(ok, start, 0)), row_seq=i32(torch.where(live, seq, -1)), row_pos=i32(torch.where(live, pos, -1)),
                slot_map=torch.where(live, slot, -1), status=i32(~ok).view(1))


def _plain_sample(s):
    z, ids = s["z"].double(), torch.arange(s["z"].shape[1], device="cuda")
    z = torch.where((ids >= s["lo"][:, None]) & (ids < s["hi"][:, None]), z, -math.inf)
    z, order = torch.sort(z, dim=-1, descending=True, stable=True)
    greedy = (s["temperature"] == 0)[:, None]
    d = (z - z[:, :1]) / torch.where(greedy, 1.0, s["temperature"].double()[:, None])
    w = d.exp()
    total = w.sum(-1, keepdim=True)
    rank = ids[None]
    k = torch.where(s["top_k"] > 0, s["top_k"], len(ids))[:, None]
    w = torch.where(rank < k, w, 0.0)
    mass = w.cumsum(-1)
    top_p = s["top_p"].double()[:, None]
    n = torch.where(top_p < 1, 1 + (mass < top_p * mass[:, -1:]).sum(-1, keepdim=True), len(ids))
    w = torch.where((rank < n) & (w >= s["min_p"].double()[:, None]) | (rank == 0), w, 0.0)
    kept = w.cumsum(-1)
    at = (kept <= s["u"].double()[:, None] * kept[:, -1:]).sum(-1, keepdim=True)
    at = torch.where(greedy, 0, torch.minimum(at, (w > 0).sum(-1, keepdim=True) - 1))
    token = order.gather(-1, at)[:, 0].to(torch.int32)
    return dict(token=token, logprob=(d.gather(-1, at) - total.log())[:, 0].float())


# ------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "map": _plain_map, "sample": _plain_sample}[kind](s)
    from paper_2603_09215_b200 import binding
    if kind == "attend":
        return binding.paged_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], row_start=s["row_start"], max_rows=s["max_rows"],
                                       max_len=s["max_len"], k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["out"])
    if kind == "append":
        binding.paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], q=s["q"], q_out=s["q_out"], row_pos=s["pos"],
                             rope=s["rope"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    if kind == "map":
        binding.page_map(s["lens"], s["rows"], s["table"], s["ring"], s["queue"], s["case"]["page"], **s["out"])
        return dict(s["out"], table=s["table"], ring=s["ring"])
    binding.sample(s["z"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                   id_lo=s["lo"], id_hi=s["hi"], token=s["token"], logprob=s["logprob"])
    return dict(token=s["token"], logprob=s["logprob"])


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    """Bytes: every input and output once (of the cache the positions that a pass reads or writes).  Flops: of attention
    four a query head, position and dimension, of the others a few a number."""
    if case["kind"] == "attend":
        lens, rows = _rows_of(case)
        q, kv = case["q_heads"] * case["head_dim"], case["kv_heads"] * case["head_dim"]
        pairs = sum(r * (n - r) + r * (r + 1) // 2 for n, r in zip(lens, rows))
        return {"bytes": 2 * sum(lens) * kv * BYTES[case["cache"]] + 2 * sum(rows) * q * BYTES[case["q"]], "flops": 4 * pairs * q}
    if case["kind"] == "append":
        q, kv, live = case["q_heads"] * case["head_dim"], case["kv_heads"] * case["head_dim"], case["rows"] - case["pad"]
        b = case["rows"] * (q * (BYTES[case["x"]] + 2) + 12 + 4 * case["head_dim"]) + 2 * live * kv * (BYTES[case["x"]] + BYTES[case["cache"]])
        return {"bytes": b, "flops": case["rows"] * 3 * (q + kv)}
    if case["kind"] == "map":
        lens, rows = _steps_of(case)
        P = case["page"]
        pages = sum(abs(-(-(n + r) // P) - -(-n // P)) if r >= 0 else -(-n // P) for n, r in zip(lens, rows))
        return {"bytes": 16 * len(lens) + 8 * pages + 16 * sum(max(r, 0) for r in rows), "flops": 4 * sum(max(r, 0) for r in rows)}
    n, ids = case["rows"], 0
    for i in range(n):
        ids += case["text"] if case["text"] > 0 and (case["speech"] == 0 or i % 3 > 0) else case["speech"]
    return {"bytes": ids * BYTES[case["x"]] + 32 * n, "flops": 8 * ids}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_attend(s):
    """Request by request, its pages laid end to end."""
    c, out = s["case"], []
    g = c["q_heads"] // c["kv_heads"]
    start, lens = s["row_start"].tolist(), s["lens"].tolist()
    for i, n in enumerate(lens):
        pages = s["table"][i, :-(-n // c["page"])].long()
        k, v = (torch.cat(list(x[pages].double()), 1)[:, :n] for x in (s["k"], s["v"]))  # [heads, n, dim]
        if s["k_scale"] is not None:
            k, v = k * s["k_scale"].double().view(-1, 1, 1), v * s["v_scale"].double().view(-1, 1, 1)
        rows = start[i + 1] - start[i]
        q = s["q"][start[i]:start[i + 1]].double().view(rows, -1, g, c["head_dim"])
        for r in range(rows):
            m = n - rows + r + 1
            p = torch.softmax(torch.einsum("hgd,hnd->hgn", q[r], k[:, :m]) / c["head_dim"] ** 0.5, -1)
            out.append(torch.einsum("hgn,hnd->hgd", p, v[:, :m]).reshape(c["q_heads"], -1))
    return torch.stack(out)


def _exact_append(s):
    """The pools as long rows of slots; every number turned as a complex one."""
    cs = torch.view_as_complex(s["rope"].double())[s["pos"].long()][:, None]

    def turned(x):
        x = x.double()
        half = x.shape[-1] // 2
        y = torch.complex(x[..., :half], x[..., half:]) * cs
        return torch.cat([y.real, y.imag], -1)

    live = s["slots"][s["slots"] >= 0]
    page, at = live // s["case"]["page"], live % s["case"]["page"]
    out = dict(q=turned(s["q"]))
    for name, x, scale in (("k_cache", turned(s["k"]), s["k_scale"]), ("v_cache", s["v"].double(), s["v_scale"])):
        new = x[:len(live)] if scale is None else x[:len(live)] / scale.double()[:, None]
        pool = s[name].double()
        most = LARGEST[s["case"]["cache"]]
        pool[page, :, at] = new if most is None else new.clamp(-most, most)
        out[name] = pool
    return out


def _exact_sample(s, drawn):
    lo, hi, T = s["lo"].tolist(), s["hi"].tolist(), s["temperature"].double()
    out = []
    for i, t in enumerate(drawn.tolist()):
        z = s["z"][i, lo[i]:hi[i]].double() / (1.0 if T[i] == 0 else T[i])
        out.append(z[t - lo[i]] - torch.logsumexp(z, 0))
    return torch.stack(out)


def _drawn(s):
    """The ids that the definition draws, row by row: the order of falling logits, cut and walked through."""
    out = []
    for i in range(len(s["u"])):
        lo, hi, T = int(s["lo"][i]), int(s["hi"][i]), float(s["temperature"][i])
        z = s["z"][i, lo:hi].double()
        z, order = torch.sort(z, dim=0, descending=True, stable=True)
        if T == 0:
            out.append(lo + int(order[0]))
            continue
        k = int(s["top_k"][i])
        p = torch.softmax(z / T, 0)
        p = p[:k] if k > 0 else p
        n = len(p)
        if float(s["top_p"][i]) < 1:
            n = 1 + int(torch.searchsorted(torch.cumsum(p, 0), float(s["top_p"][i]) * p.sum()))
        n = min(n, max(1, int((p >= float(s["min_p"][i]) * p[0]).sum())))
        n = max(1, min(n, int((p > 0).sum())))
        c = torch.cumsum(p[:n], 0)
        j = int(torch.searchsorted(c, float(s["u"][i]) * c[-1], right=True))
        out.append(lo + int(order[min(j, n - 1)]))
    return torch.tensor(out)


def exact(case, seed):
    if case["kind"] == "map":
        return None
    s = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(s)
    if case["kind"] == "append":
        return _exact_append(s)
    return dict(token=None, logprob=_exact_sample(s, _drawn(s)))
