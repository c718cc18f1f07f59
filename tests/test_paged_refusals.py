"""What the paged operators refuse: found from the arguments alone, before anything is launched (no GPU needed).  The addresses
are never followed."""
import ctypes

import pytest
import torch

from paper_2603_09215_b200 import binding as B

A = 1 << 20  # an aligned address


def call(name, a):
    return getattr(B.load(), name)(ctypes.addressof(a), None)


def map_args(**kw):
    v = dict(seq_len=A, seq_rows=A + 4096, block_table=A, ring=A, queue=A + 8192, seq_len_out=A + 12288, queue_out=A + 16384, row_start=A,
             row_seq=A, row_pos=A, slot_map=A, status=A, table_stride=9, n_seqs=4, max_blocks=9, page_size=16, ring_size=5, max_rows=6)
    v.update(kw)
    return B.PageMapArgs(**v)


@pytest.mark.parametrize("bad", [
    {k: None} for k in ("seq_len", "seq_rows", "block_table", "ring", "queue", "seq_len_out", "queue_out", "row_start", "row_seq", "row_pos",
                        "slot_map", "status")] + [
    dict(n_seqs=0), dict(n_seqs=-1), dict(max_blocks=0), dict(page_size=0), dict(ring_size=0), dict(max_rows=-1), dict(table_stride=8),
    dict(slot_map=A + 4), dict(ring=A + 2), dict(queue_out=A + 8192), dict(queue_out=A + 8196), dict(seq_len_out=A), dict(seq_len_out=A + 12),
    dict(seq_len_out=A + 4096), dict(queue_out=A + 4)])
def test_page_map_refuses(bad):
    assert call("sparsk_page_map", map_args(**bad)) == B.EINVAL


def test_page_map_refuses_more_sequences_than_it_holds():
    far = dict(seq_rows=A << 1, queue=A << 2, seq_len_out=A << 3, queue_out=A << 4)
    assert call("sparsk_page_map", map_args(n_seqs=12289, **far)) == B.ECAPACITY
    assert B.load().sparsk_page_map(None, None) == B.EINVAL


def pool(**kw):
    v = dict(k=A, v=A, page_stride=16 * 128, head_stride=16 * 64, pos_stride=64, type=B.FP16, n_pages=3, n_kv_heads=2, page_size=16, head_dim=64)
    v.update(kw)
    return B.PagePool(**v)


BAD_POOLS = [dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(k_scale=A + 2), dict(type=B.FP32), dict(type=7), dict(head_dim=96),
             dict(n_pages=0), dict(n_kv_heads=0), dict(page_size=0), dict(page_stride=2044), dict(head_stride=-64), dict(pos_stride=68),
             dict(pos_stride=32), dict(page_stride=1 << 31)]


def append_args(pool_kw={}, **kw):
    v = dict(pool=pool(**pool_kw), k=A, v=A, q=A, q_out=A, slot_map=A, row_pos=A, rope=A, k_row_stride=128, k_head_stride=64, v_row_stride=128,
             v_head_stride=64, q_row_stride=256, q_head_stride=64, q_out_row_stride=256, q_out_head_stride=64, x_type=B.BF16, q_out_type=B.BF16,
             n_rows=0, n_q_heads=4, rope_len=8)
    v.update(kw)
    return B.PagedAppendArgs(**v)


@pytest.mark.parametrize("bad", [dict(pool_kw=p) for p in BAD_POOLS] + [
    dict(k=None), dict(v=None), dict(slot_map=None), dict(slot_map=A + 4), dict(k=A + 1), dict(x_type=B.E4M3), dict(x_type=-1), dict(q_out=None),
    dict(q_out_type=B.FP32), dict(n_q_heads=0), dict(n_rows=-1), dict(k_row_stride=-1), dict(v_head_stride=1 << 30), dict(q_row_stride=-4),
    dict(q_out_head_stride=-1), dict(row_pos=None), dict(rope_len=0), dict(rope=A + 2), dict(x_type=B.FP32, q=A + 2)])
def test_append_refuses(bad):
    assert call("sparsk_paged_append", append_args()) == B.OK  # (no rows: nothing to launch)
    assert call("sparsk_paged_append", append_args(**bad)) == B.EINVAL


def attn_args(pool_kw={}, **kw):
    v = dict(pool=pool(**pool_kw), q=A, out=A, block_table=A, seq_len=A, row_start=A, table_stride=7, q_row_stride=256, q_head_stride=64,
             out_row_stride=256, out_head_stride=64, q_type=B.BF16, n_rows=0, n_seqs=2, max_blocks=7, n_q_heads=4, max_rows=1, max_len=50)
    v.update(kw)
    return B.PagedAttnArgs(**v)


def attend(a, scratch=A, nbytes=1 << 40):
    return B.load().sparsk_paged_attention(ctypes.addressof(a), scratch, nbytes, None)


@pytest.mark.parametrize("bad", [dict(pool_kw=p) for p in BAD_POOLS + [dict(page_size=8), dict(page_size=24), dict(type=B.BF16)]] + [
    dict(q_type=B.FP32), dict(q_type=B.E4M3), dict(n_rows=-1), dict(n_seqs=0), dict(max_blocks=0), dict(n_q_heads=3), dict(n_q_heads=0),
    dict(max_rows=-1), dict(max_len=-1), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(table_stride=6),
    dict(max_blocks=1 << 28, table_stride=1 << 28), dict(row_start=None), dict(q_row_stride=-1), dict(out_head_stride=1 << 30)])
def test_attention_refuses(bad):
    assert attend(attn_args()) == B.OK  # (no rows)
    if bad == dict(pool_kw=dict(type=B.BF16)):
        bad = dict(bad, q_type=B.FP16)  # 16-bit queries of more precision than the pool's
    a = attn_args(**bad)
    assert attend(a) == B.EINVAL and B.load().sparsk_paged_attention_scratch_bytes(ctypes.addressof(a)) == 0


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(block_table=None), dict(seq_len=None), dict(q=A + 1), dict(lse=A + 2),
                                 dict(seq_len=A + 1)])
def test_attention_refuses_addresses(bad):
    assert attend(attn_args(**bad)) == B.EINVAL


def test_attention_refuses_scratch():
    assert attend(attn_args(), None) == attend(attn_args(), A + 16) == attend(attn_args(), A, 8) == B.EINVAL


def sample_args(**kw):
    v = dict(logits=A, uniforms=A, token=A, row_stride=50, type=B.FP32, n_rows=2, n_ids=50)
    v.update(kw)
    return B.SampleArgs(**v)


@pytest.mark.parametrize("bad,code", [(dict(logits=None), -1), (dict(uniforms=None), -1), (dict(token=None), -1), (dict(type=B.E4M3), -1),
                                      (dict(n_rows=0), -1), (dict(n_ids=0), -1), (dict(row_stride=-1), -1), (dict(logits=A + 2), -1),
                                      (dict(top_k=A + 2), -1), (dict(logprob=A + 1), -1), (dict(n_ids=262145), -2)])
def test_sample_refuses(bad, code):
    assert call("sparsk_sample", sample_args(**bad)) == code


def test_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros((2, 1, 16, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    for f in (lambda: B.page_map(i, i, x, i, i, 16, max_rows=2), lambda: B.paged_append(x[:, :, 0], x[:, :, 0], x, x, i),
              lambda: B.paged_attention(x[:, :, 0], x, x, i.view(1, 2), i), lambda: B.sample(torch.zeros((2, 5)), torch.zeros(2))):
        with pytest.raises(B.SparskError) as e:
            f()
        assert e.value.code == B.EINVAL


def test_binding_refuses_what_is_not_a_tensor():
    x = torch.zeros((2, 1, 16, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    for f in (lambda: B.paged_append([1], x[:, :, 0], x, x, i), lambda: B.paged_attention(x[:, :, 0], None, x, i.view(1, 2), i, out=x[:, :, 0]),
              lambda: B.page_map(i, i, x, i, i, 16), lambda: B.sample(5, i, token=i),
              lambda: B.page_map(7, i, x, i, i, 16, seq_len=i, queue=i, row_start=i, row_seq=i, row_pos=i, slot_map=i, status=i)):
        with pytest.raises(B.SparskError) as e:
            f()
        assert e.value.code == B.EINVAL
    with pytest.raises(TypeError):
        B._native().sample(x)
