"""Host-side checks of the paged cache's C ABI that need no GPU: structures, argument rejection, size arithmetic."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from paper_2510_18716_b200 import binding as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ssd_b200.h")
BUF = np.zeros(4096, np.uint8)
AT = (BUF.ctypes.data + 255) // 256 * 256          # never dereferenced: every call below is refused before a launch


@pytest.mark.parametrize("name,struct", [("ssd_paged_kv", B.SsdPagedKv), ("ssd_paged_attn", B.SsdPagedAttn)])
def test_struct_matches_header(name, struct):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    kinds = {"int64_t": C.c_int64, "int32_t": C.c_int32, "float": C.c_float, "size_t": C.c_size_t}
    want = []
    for decl in body.split(";"):
        decl = " ".join(decl.replace("const", "").split())
        if not decl:
            continue
        kind, rest = decl.split(" ", 1)
        for field in rest.split(","):
            field = field.strip()
            want.append((field.lstrip("*").strip(), C.c_void_p if field.startswith("*") else kinds[kind]))
    assert [(n, t) for n, t in struct._fields_] == want


def kv(**change):
    d = dict(k_pages=AT, v_pages=AT, k_scales=None, v_scales=None, page_table=AT, lengths=AT, scores=AT, status=None, page_stride=8 * 16 * 128,
             head_stride=16 * 128, slot_stride=128, table_seq_stride=4, len_seq_stride=8, len_head_stride=1, score_seq_stride=512,
             score_head_stride=64, dtype=0, n_seqs=2, n_kv_heads=8, head_dim=128, page_size=16, n_pages=9, max_pages=4, score_slots=64)
    d.update(change)
    return B.SsdPagedKv(**d)


def attn(**change):
    d = dict(q=AT, out=AT, k_new=AT, v_new=AT, lse=None, workspace=AT, workspace_bytes=1 << 30, q_seq_stride=1024, q_head_stride=128,
             out_seq_stride=1024, out_head_stride=128, new_seq_stride=1024, new_head_stride=128, q_dtype=0, n_q_heads=8, accumulate=0,
             softmax_scale=0.0)
    d.update(change)
    return B.SsdPagedAttn(**d)


BAD_VIEWS = [dict(k_pages=None), dict(v_pages=None), dict(page_table=None), dict(lengths=None), dict(k_pages=AT + 8), dict(page_table=AT + 2),
             dict(lengths=AT + 1), dict(scores=AT + 2), dict(dtype=3), dict(dtype=-1), dict(head_dim=96), dict(head_dim=0), dict(n_seqs=-1),
             dict(n_kv_heads=0), dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(slot_stride=124), dict(page_stride=-128),
             dict(head_stride=1 << 60), dict(table_seq_stride=-1), dict(len_head_stride=-1), dict(score_slots=0), dict(k_scales=AT),
             dict(dtype=2), dict(dtype=2, k_scales=AT), dict(dtype=2, k_scales=AT, v_scales=AT, slot_stride=120)]
LARGE_VIEWS = [dict(n_kv_heads=129), dict(max_pages=1 << 26), dict(max_pages=1 << 30, page_size=64), dict(n_seqs=1 << 22)]


@pytest.mark.parametrize("change,code", [(c, B.SSD_ERR_INVALID_ARG) for c in BAD_VIEWS] + [(c, B.SSD_ERR_LIMIT) for c in LARGE_VIEWS])
def test_bad_views_are_refused_by_every_call(change, code):
    lib, view = B.load(), kv(**change)
    ints = (C.c_int32 * 129)(*([1] * 129))
    a = attn(n_q_heads=max(1, view.n_kv_heads))
    before = B.kernel_launch_count()
    assert lib.ssd_paged_append(view, AT, AT, 0, 1024, 128, None, view.n_seqs, None) == code
    assert lib.ssd_paged_decode_attn(view, a, None) == code
    assert lib.ssd_paged_append_decode(view, a, None) == code
    assert lib.ssd_paged_evict(view, None, 0, ints, ints, AT, 64, AT, None) == code
    assert lib.ssd_paged_workspace_bytes(view, 8, 0) == 0
    assert B.kernel_launch_count() == before


@pytest.mark.parametrize("change", [
    dict(q=None), dict(out=None), dict(workspace=None), dict(q=AT + 2), dict(out=AT + 8), dict(workspace=AT + 16), dict(lse=AT + 2), dict(q_dtype=1),
    dict(q_dtype=2), dict(n_q_heads=12), dict(n_q_heads=0), dict(n_q_heads=-8), dict(q_head_stride=4), dict(out_seq_stride=-1024),
    dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf"))])
def test_bad_attention_arguments(change):
    lib = B.load()
    assert lib.ssd_paged_decode_attn(kv(), attn(**change), None) == B.SSD_ERR_INVALID_ARG
    assert lib.ssd_paged_append_decode(kv(), attn(**change), None) == B.SSD_ERR_INVALID_ARG


def test_more_query_heads_than_can_be_counted():
    lib = B.load()
    many = 8 << 26
    assert lib.ssd_paged_decode_attn(kv(), attn(n_q_heads=many), None) == B.SSD_ERR_LIMIT
    assert lib.ssd_paged_append_decode(kv(max_pages=1 << 20), attn(n_q_heads=8 << 16), None) == B.SSD_ERR_LIMIT


def test_bad_arguments_of_single_calls():
    lib = B.load()
    bad = B.SSD_ERR_INVALID_ARG
    assert lib.ssd_paged_decode_attn(None, attn(), None) == bad and lib.ssd_paged_decode_attn(kv(), None, None) == bad
    assert lib.ssd_paged_decode_attn(kv(scores=None), attn(accumulate=1), None) == bad
    for c in (dict(k_new=None), dict(v_new=None), dict(k_new=AT + 4), dict(new_head_stride=12)):
        assert lib.ssd_paged_append_decode(kv(), attn(**c), None) == bad
    append = lambda view=kv(), k=AT, v=AT, t=0, ts=1024, hs=128, cu=None, n=2: lib.ssd_paged_append(view, k, v, t, ts, hs, cu, n, None)  # noqa: E731
    assert append(k=None) == append(v=None) == append(k=AT + 2) == append(t=1) == append(t=2) == append(ts=-8) == append(hs=4) == bad
    assert append(n=3) == append(n=-1) == append(cu=AT + 2, n=3) == append(view=None) == bad
    assert append(cu=AT, n=0, k=None, v=None) == B.SSD_OK            # a step without new tokens
    ints = lambda x: (C.c_int32 * 8)(*([x] * 8))  # noqa: E731

    def evict(view=None, into=None, prefix=4, b=ints(8), r=ints(4), kept=AT, cols=16, counts=AT):
        return lib.ssd_paged_evict(view or kv(), into, prefix, b, r, kept, cols, counts, None)
    assert evict(view=kv(scores=None)) == evict(prefix=-1) == evict(b=None) == evict(r=None) == evict(kept=None) == evict(counts=None) == bad
    assert evict(b=ints(-1)) == evict(r=ints(-1)) == evict(cols=15) == evict(cols=0) == evict(kept=AT + 2) == bad
    assert evict(b=ints(0x7fffffff)) == B.SSD_ERR_LIMIT
    # one length per sequence and different budgets; another type, shape or the same tables as the target
    uneven = (C.c_int32 * 8)(*range(8))
    assert evict(view=kv(len_head_stride=0), b=uneven) == bad
    other = dict(page_table=AT + 64, lengths=AT + 128, scores=AT + 256)
    for c in (dict(dtype=1), dict(head_dim=64), dict(n_kv_heads=4), dict(n_seqs=1), dict(max_pages=0), dict(page_table=AT), dict(lengths=AT),
              dict(scores=AT), dict(page_size=1, page_stride=1024, max_pages=15)):
        assert evict(into=kv(**{**other, **c})) == bad


def test_writes_through_broadcast_strides_are_refused():
    """What a call writes needs places of its own; what it only reads may be broadcast (here: up to a later refusal)."""
    lib, bad = B.load(), B.SSD_ERR_INVALID_ARG
    ints = (C.c_int32 * 8)(*([4] * 8))
    other = dict(page_table=AT + 64, lengths=AT + 128, scores=AT + 256)
    q8 = dict(dtype=2, k_scales=AT, v_scales=AT, scale_page_stride=128, scale_head_stride=16, scale_slot_stride=1)
    pages = [dict(page_stride=0), dict(head_stride=0), dict(slot_stride=0), dict(table_seq_stride=0)]
    pages += [{**q8, x: 0} for x in ("scale_page_stride", "scale_head_stride", "scale_slot_stride")]
    scores = [dict(score_seq_stride=0), dict(score_head_stride=0)]
    for c in pages + scores:
        view = kv(**c)
        assert lib.ssd_paged_append(view, AT, AT, 0, 1024, 128, None, 2, None) == bad
        assert lib.ssd_paged_append_decode(view, attn(), None) == bad
        assert lib.ssd_paged_evict(view, None, 4, ints, ints, AT, 12, AT, None) == bad
        assert lib.ssd_paged_evict(kv(**{k: x for k, x in c.items() if k in q8}), kv(**{**other, **c}), 4, ints, ints, AT, 12, AT, None) == bad
    for c in scores:
        assert lib.ssd_paged_decode_attn(kv(**c), attn(accumulate=1), None) == bad
    assert lib.ssd_paged_evict(kv(len_seq_stride=0), None, 4, ints, ints, AT, 12, AT, None) == bad
    assert lib.ssd_paged_evict(kv(), kv(**other, len_seq_stride=0), 4, ints, ints, AT, 12, AT, None) == bad
    for c in (dict(out_seq_stride=0), dict(out_head_stride=0)):
        assert lib.ssd_paged_decode_attn(kv(), attn(**c), None) == bad
    # one of something has no stride, a table per head makes its pages the head's own, and an empty step writes nothing
    one = kv(n_seqs=1, table_seq_stride=0, score_seq_stride=0, table_head_stride=4, head_stride=0)
    assert lib.ssd_paged_append(one, AT, AT, 0, 1024, 128, AT, 0, None) == B.SSD_OK


def test_head_budgets_follow_the_labels():
    b, r = B.head_budgets([1, 0, 0, 1], window=64, sink_budget=96, sink_recent=24)
    assert b == [96, 0, 0, 96] and r == [24, 64, 64, 24]


def test_the_handle_refuses_what_is_not_on_a_gpu():
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.PagedKV(k, k, t, n)
    with pytest.raises(ValueError, match="head_dim"):
        B.PagedKV(k.float(), k.float(), t, n)
    with pytest.raises(ValueError, match="page_table"):
        B.PagedKV(k, k, t.long(), n)
    with pytest.raises(ValueError, match="lengths"):
        B.PagedKV(k, k, t, n.float())
    with pytest.raises(ValueError, match="scales"):
        B.PagedKV(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), t, n)
    with pytest.raises(ValueError, match="strides"):
        B.PagedKV(k, k.transpose(1, 2).contiguous().transpose(1, 2), t, n)
    with pytest.raises(ValueError, match="scores"):
        B.PagedKV(k, k, t, n, scores=torch.zeros(1, 3, 8))
    with pytest.raises(ValueError, match="heads"):
        B.PagedKV(k, k, torch.zeros(1, 4, 2, dtype=torch.int32), n)
    with pytest.raises(ValueError, match="empty"):
        B.PagedKV(k, k, torch.zeros(0, 2, dtype=torch.int32), torch.zeros(0, dtype=torch.int32))
