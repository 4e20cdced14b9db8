"""GPU parity of the paged cache against plain float64 arithmetic, element by element.

Tolerances.  With u = 2^-24, D the head dimension, n the slots, x = scale q.k and A = max over slots of scale sum |q||k|:
a logit is a sum of D exact products in float32, each of the D additions off by at most 2^-23 of the partial sums (the
products' unit truncates): |dx| <= D 2^-23 A, and its scaling and the subtraction of the maximum add 4 u (|x| + |m|),
both below 8 u A, and 16 u for the constant 2^14 that the weights carry (14 / 2^k steps of u).  e^x adds 2^-22, the two-term
rounding of a weight 2^-17 (bf16: 2^-9 twice, and a margin of two; fp16 less; over 8-bit pages, with a bf16 result, a
weight is one fp16 number, whose rounding is off by 2^-11 at most), the sums over n slots at most n u relative to
the sum of the absolute terms, merging and the final division 2^-21.  So a weight is off by at most
    delta = D 2^-23 A + 8 u A + 2^-17 (8 bits to bf16: 2^-11) + n u + 2^-20     (relative)
and twice that after the division by the sum, which has the same error.  In fp16 (fp16 and 8-bit pages) a weight also has an
absolute error: the largest is held at 2^14, the smallest step is 2^-24, so half a step is 2^-39 of the largest; with a margin
of two an output is off by 2^-38 max(w) sum |v| on that account (8 bits: 2^-38 max(w scale) sum |code|, the scale being part
of the weight there).  An output is off by 2 delta sum w |v|, that, and its own rounding, half a step: eps/2 |o|.  An accumulated score is off by 2 delta of the weights added and u of its value for each
of the g + 1 additions; a log of the sum by delta and 4 u of its value.
"""
import math

import numpy as np
import pytest
import torch

from paper_2510_18716_b200 import binding as B
from paper_2510_18716_b200 import workloads as wl

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
U = 2.0 ** -24


def dev():
    return torch.device("cuda:0")


class Paged:
    """A cache with poisoned unused slots, its handle, and its rows in float64."""

    def __init__(self, lens, heads, d=128, dtype="bf16", page=16, order="head", per_head=False, scores=False, seed=0, room=0, spare=3):
        lens = np.asarray(lens, np.int64)
        self.n = np.broadcast_to(lens[:, None], (len(lens), heads)).copy() if lens.ndim == 1 else lens
        self.heads, self.d, self.dtype, self.page, self.per_head = heads, d, dtype, page, per_head
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = self.n if per_head else self.n.max(axis=1, keepdims=True)
        need = -(-(rows + room) // page)
        self.max_pages = max(1, int(need.max()))
        n_pages = int(need.sum()) + spare
        pool = 1 if per_head else heads
        shape = (n_pages, pool, page, d) if order == "head" else (n_pages, page, pool, d)
        perm = torch.randperm(n_pages, generator=g, device="cuda").cpu().numpy()
        table = np.full((len(lens), rows.shape[1], self.max_pages), -1, np.int32)
        at = 0
        for i in range(len(lens)):
            for h in range(rows.shape[1]):
                table[i, h, : need[i, h]] = perm[at: at + need[i, h]]
                at += need[i, h]
        self.table_np = table
        self.table = torch.from_numpy(table if per_head else table[:, 0]).cuda()
        ln = self.n if (per_head or lens.ndim == 2) else self.n[:, 0]
        self.lengths = torch.from_numpy(np.ascontiguousarray(ln).astype(np.int32)).cuda()
        held = torch.zeros((n_pages, pool, page), dtype=torch.bool)
        for i in range(len(lens)):
            for h in range(heads):
                s = np.arange(self.n[i, h])
                held[table[i, h % table.shape[1]][s // page], h % pool, s % page] = True
        held = held.cuda()
        self.pages, self.scales = [], []
        for _ in range(2):
            x = torch.randn(shape, generator=g, device="cuda")
            x = x if order == "head" else x.transpose(1, 2)
            sc = None
            if dtype == "e4m3":
                sc = torch.rand((n_pages, pool, page), generator=g, device="cuda") * 0.02 + 1e-4
                sc = torch.where(held, sc, torch.full_like(sc, math.nan))
                x = (x * 100.0).clamp(-448.0, 448.0)                         # beyond, the conversion makes NaN codes
            x = torch.where(held[..., None], x, torch.full_like(x, math.nan))       # what must not be read
            self.pages.append(x.to(TYPES[dtype]))
            self.scales.append(sc)
        self.scores = None
        if scores:
            self.scores = torch.exp(torch.randn((len(lens), heads, self.max_pages * page), generator=g, device="cuda"))
        self.kv = B.PagedKV(self.pages[0], self.pages[1], self.table, self.lengths, k_scales=self.scales[0], v_scales=self.scales[1],
                            scores=self.scores)

    def rows(self, which, i, h, n=None):
        """The first n rows of a head, float64 [n, D]."""
        n = int(self.n[i, h]) if n is None else n
        s = np.arange(n)
        pg = torch.from_numpy(self.table_np[i, h % self.table_np.shape[1]][s // self.page].astype(np.int64)).cuda()
        r, hh = torch.from_numpy(s % self.page).cuda(), h % self.pages[which].shape[1]
        x = self.pages[which].view(torch.uint8)[pg, hh, r].view(self.pages[which].dtype) if self.dtype == "e4m3" else self.pages[which][pg, hh, r]
        x = x.double()
        return x if self.dtype != "e4m3" else x * self.scales[which][pg, hh, r].double()[:, None]

    def row_scales(self, i, h):
        """V's scales of a head."""
        s = np.arange(int(self.n[i, h]))
        pg = torch.from_numpy(self.table_np[i, h % self.table_np.shape[1]][s // self.page].astype(np.int64)).cuda()
        return self.scales[1][pg, h % self.pages[1].shape[1], torch.from_numpy(s % self.page).cuda()].double().clamp(min=1e-300)

    def bits(self):
        got = [p.contiguous().view(torch.uint8).clone() for p in self.pages]
        return got + [s.contiguous().view(torch.uint8).clone() for s in self.scales if s is not None]


def reference(c, q, scale=None):
    """(out, lse, weights [n_seqs, heads, slots], and the bounds on the errors of the three) in float64."""
    scale = 1.0 / math.sqrt(c.d) if scale is None else scale
    n_seqs, hq = q.shape[:2]
    g = hq // c.heads
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full((n_seqs, hq), -math.inf, dtype=torch.float64, device="cuda")
    w_all = torch.zeros((n_seqs, c.heads, c.max_pages * c.page), dtype=torch.float64, device="cuda")
    e_out, e_lse, e_w = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(w_all)
    half = torch.finfo(q.dtype).eps / 2
    for i in range(n_seqs):
        for h in range(c.heads):
            n = int(c.n[i, h])
            if n == 0:
                continue
            k, v = c.rows(0, i, h), c.rows(1, i, h)
            qq = q[i, h * g:(h + 1) * g].double()
            x = scale * qq @ k.T
            a = (scale * qq.abs() @ k.abs().T).amax(dim=1, keepdim=True)
            m = x.amax(dim=1, keepdim=True)
            e = (x - m).exp()
            z = e.sum(dim=1, keepdim=True)
            w = e / z
            delta = c.d * 2.0 ** -23 * a + 8 * U * a + (2.0 ** -11 if c.dtype == "e4m3" and q.dtype == torch.bfloat16 else 2.0 ** -17) + n * U + 2.0 ** -20
            o = w @ v
            out[i, h * g:(h + 1) * g] = o
            floor = 0.0
            if c.dtype == "fp16":
                floor = 2.0 ** -38 * w.amax(dim=1, keepdim=True) * v.abs().sum(dim=0)
            elif c.dtype == "e4m3":
                s = c.row_scales(i, h)
                floor = 2.0 ** -38 * (w * s).amax(dim=1, keepdim=True) * (v / s[:, None]).abs().sum(dim=0)
            e_out[i, h * g:(h + 1) * g] = half * o.abs() + 2 * delta * (w @ v.abs()) + floor + torch.finfo(q.dtype).tiny
            lse[i, h * g:(h + 1) * g] = (m + z.log())[:, 0]
            e_lse[i, h * g:(h + 1) * g] = (delta + 4 * U * ((m + z.log()).abs() + 16))[:, 0]
            w_all[i, h, :n] = w.sum(dim=0)
            e_w[i, h, :n] = (2 * delta * w).sum(dim=0)
    return out, lse, w_all, e_out, e_lse, e_w


def check_attention(c, q, got, lse, scale=None, before=None):
    out, want_lse, w, e_out, e_lse, e_w = reference(c, q, scale)
    err = (got.double() - out).abs()
    ok = bool((err <= e_out).all())
    assert ok, f"out: worst {float((err / e_out.clamp(min=1e-300)).max())} of the bound"
    empty = torch.isinf(want_lse)
    assert bool((lse[empty] == -math.inf).all()) and bool((got[empty] == 0).all())
    err = torch.where(empty, torch.zeros_like(want_lse), (lse.double() - want_lse).abs())
    assert bool((err <= e_lse).all()), "lse"
    if before is not None:
        g = q.shape[1] // c.heads
        n = torch.from_numpy(c.n).cuda()[..., None]
        held = torch.arange(w.shape[2], device="cuda") < n
        want = before.double() + w
        err = (c.scores.double() - want).abs()
        ok = err <= e_w + (g + 1) * U * want.abs()
        assert bool(ok[held].all()), "scores"
        assert torch.equal(c.scores[~held], before[~held])           # what lies behind the last slot stays as it was
    assert c.kv.device_status() == 0


def new_q(c, g, seed=1, dtype=None):
    t = TYPES[dtype or (c.dtype if c.dtype != "e4m3" else "bf16")]
    return (1.5 * torch.randn((c.n.shape[0], c.heads * g, c.d), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")).to(t)


EDGE = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300]


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 3, 8, 9, 16, 20])
def test_types_dims_and_groups(dtype, d, g):
    c = Paged(EDGE, 2, d=d, dtype=dtype, scores=True, seed=g)
    q, before = new_q(c, g), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)
    assert torch.equal(c.kv.decode_attn(q), out)                     # the same bits, with and without the weights


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 256])
@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pages_and_orders(page, order, dtype):
    c = Paged(EDGE, 3, dtype=dtype, page=page, order=order, scores=True, seed=page)
    q, before = new_q(c, 2), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
def test_tables_and_lengths_of_every_head(dtype):
    n = np.random.RandomState(3).randint(0, 200, size=(9, 5))
    n[2] = 0
    c = Paged(n, 5, dtype=dtype, per_head=True, scores=True)
    q, before = new_q(c, 4, dtype="fp16" if dtype != "bf16" else "bf16"), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)
    shared = Paged(n, 5, dtype=dtype)                                # lengths of every head over a shared table
    q = new_q(shared, 4)
    out, lse = shared.kv.decode_attn(q, return_lse=True)
    check_attention(shared, q, out, lse)


@pytest.mark.parametrize("n_seqs,heads,top,g,dtype", [(40, 16, 90, 1, "bf16"), (301, 1, 70, 8, "fp16"), (64, 32, 260, 1, "e4m3"),
                                                      (3, 100, 500, 2, "bf16"), (70, 5, 333, 9, "e4m3")])
def test_many_heads(n_seqs, heads, top, g, dtype):
    n = np.random.RandomState(top).randint(0, top + 1, size=n_seqs)
    c = Paged(n, heads, dtype=dtype, scores=True, page=32)
    q, before = new_q(c, g), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)


@pytest.mark.parametrize("n,heads,g,dtype,d", [(40000, 2, 4, "bf16", 128), (9001, 1, 16, "fp16", 64), (70001, 1, 12, "e4m3", 128), (30011, 3, 1, "e4m3", 64)])
def test_long_rows_are_split_and_joined(n, heads, g, dtype, d):
    c = Paged([n], heads, d=d, dtype=dtype, scores=True, page=48)
    q, before = new_q(c, g), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)
    for _ in range(3):
        again, lse2 = c.kv.decode_attn(q, return_lse=True)
        assert torch.equal(again, out) and torch.equal(lse, lse2)    # the order of arrival does not show


def test_one_long_sequence_among_short_ones():
    c = Paged([5, 0, 20000, 1, 17] + [40] * 90, 4, scores=True)
    q, before = new_q(c, 3), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)


@pytest.mark.parametrize("n_seqs,heads,per_head", [(3000, 4, False), (700, 5, True)])
def test_more_sequences_than_threads(n_seqs, heads, per_head):
    r = np.random.RandomState(n_seqs)
    n = r.randint(0, 40, size=(n_seqs, heads) if per_head else n_seqs) * r.randint(0, 2, size=(n_seqs, 1) if per_head else n_seqs)
    c = Paged(n, heads, d=64, per_head=per_head, scores=True, page=8)
    q, before = new_q(c, 2), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    # plain arithmetic for all of them at once, on the cache's rows padded to the longest
    top = int(c.n.max())
    slot = torch.arange(top, device="cuda").expand(n_seqs, heads, -1)
    table = torch.from_numpy(np.broadcast_to(c.table_np, (n_seqs, heads, c.table_np.shape[2])).astype(np.int64)).cuda()
    held = slot < torch.from_numpy(c.n).cuda()[..., None]
    at = (torch.gather(table, 2, slot // 8).clamp(min=0), torch.arange(c.pages[0].shape[1], device="cuda").view(1, -1, 1).expand_as(slot), slot % 8)
    k, v = (torch.where(held[..., None], p[at].double(), torch.zeros((), dtype=torch.float64, device="cuda")) for p in c.pages)
    x = q.double().view(n_seqs, heads, 2, 64) @ k.transpose(2, 3) / 8.0
    x = torch.where(held[:, :, None], x, torch.full_like(x, -math.inf))
    w = torch.nan_to_num(torch.softmax(x, dim=3), nan=0.0)
    want = (w @ v).view(n_seqs, 2 * heads, 64)
    # A <= |q| |k| scale <= 50 here: delta <= 64 2^-23 50 + .. < 5e-4
    bound = 2.0 ** -8 * want.abs() + 1e-3 * (w @ v.abs()).view(n_seqs, 2 * heads, 64) + 1e-30
    assert bool(((out.double() - want).abs() <= bound).all())
    err = (c.scores[..., :top].double() - before[..., :top].double() - w.sum(dim=2)).abs()
    assert bool((err <= 1e-3 * w.sum(dim=2) + 4 * U * before[..., :top].abs() + 1e-12).all())
    assert c.kv.device_status() == 0


@pytest.mark.parametrize("g,n_seqs", [(128, 3), (40, 30)])
def test_very_large_groups(g, n_seqs):
    c = Paged([200, 17, 90] * (n_seqs // 3), 1, scores=True)
    q, before = new_q(c, g), c.scores.clone()
    out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)


def test_all_sequences_empty():
    c = Paged([0, 0, 0], 4, scores=True)
    q, before = new_q(c, 2), c.scores.clone()
    out, lse = c.kv.decode_attn(q, out=torch.full_like(q, math.nan), return_lse=True, accumulate=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all()) and torch.equal(c.scores, before)
    bits = c.bits()
    c.kv.append_decode(q[:, :4].contiguous(), q[:, :4].contiguous(), q)
    assert all(torch.equal(a, b) for a, b in zip(bits, c.bits())) and c.kv.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
def test_large_logits_and_scales(dtype):
    """Logits of some hundred and rows of very different size: weights from one slot only down to nothing."""
    c = Paged([400, 33, 1000], 2, dtype=dtype, seed=5)
    if dtype == "e4m3":
        g = torch.Generator(device="cuda").manual_seed(29)
        c.scales[1].mul_(torch.exp2(torch.randint(-40, 20, c.scales[1].shape, generator=g, device="cuda").float()))
    q = new_q(c, 4) * 64
    out, lse = c.kv.decode_attn(q, return_lse=True)
    check_attention(c, q, out, lse)
    for s in (0.0, 0.001, 2.5):
        kv = B.PagedKV(c.pages[0], c.pages[1], c.table, c.lengths, k_scales=c.scales[0], v_scales=c.scales[1], softmax_scale=s)
        small = new_q(c, 4, seed=9)
        out, lse = kv.decode_attn(small, return_lse=True)
        check_attention(c, small, out, lse, scale=s or None)


def test_strided_queries_and_outputs():
    c = Paged([70, 5, 0, 33], 4, scores=True)
    fused = torch.randn((4, 8 + 4 + 4, 128), device="cuda").to(torch.bfloat16)       # q, k, v of a projection
    q = fused[:, :8]
    big = torch.full((4, 10, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[:, 1:9, :128]
    before = c.scores.clone()
    got, lse = c.kv.decode_attn(q, out=out, return_lse=True, accumulate=True)
    check_attention(c, q, out, lse, before=before)
    assert bool((big[:, 0] == 7).all()) and bool((big[:, 9] == 7).all()) and bool((big[..., 128:] == 7).all())
    turned = torch.randn((8, 4, 128), device="cuda").to(torch.bfloat16).transpose(0, 1)     # heads first in memory
    out, lse = c.kv.decode_attn(turned, return_lse=True)
    check_attention(c, turned, out, lse)


def test_offsets_beyond_32_bits():
    """Pages 3 GB apart."""
    far = 3 * (1 << 29) + 4096                                       # elements of 2 bytes
    raw = torch.empty(far * 2 + (1 << 20), dtype=torch.bfloat16, device="cuda")
    shape, strides = (3, 2, 16, 128), (far, 2048, 128, 1)
    k = raw.as_strided(shape, strides)
    v = raw.as_strided(shape, strides, 8192)
    g = torch.Generator(device="cuda").manual_seed(2)
    for x in (k, v):
        x.copy_(torch.randn(shape, generator=g, device="cuda"))
    c = Paged([48, 20], 2)
    c.pages = [k, v]
    c.table_np = np.array([[[2, 0, 1]], [[1, 2, -1]]], np.int32)
    c.table = torch.from_numpy(c.table_np[:, 0]).cuda()
    c.kv = B.PagedKV(k, v, c.table, c.lengths)
    q = new_q(c, 2)
    out, lse = c.kv.decode_attn(q, return_lse=True)
    check_attention(c, q, out, lse)


# ------------------------------------------------------------------------------------------------ device data that is wrong
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pages_outside_the_pool_are_masked(dtype):
    c = Paged([100, 40, 16], 2, dtype=dtype, scores=True)
    bad = c.table.clone()
    bad[0, 3] = 10 ** 6
    bad[1, 0] = -7
    bad[2, 0] = c.pages[0].shape[0]
    kv = B.PagedKV(c.pages[0], c.pages[1], bad, c.lengths, k_scales=c.scales[0], v_scales=c.scales[1], scores=c.scores)
    q, before = new_q(c, 2), c.scores.clone()
    out, lse = kv.decode_attn(q, return_lse=True, accumulate=True)
    assert kv.device_status() == 1
    # the same cache without the masked slots
    good = Paged([84, 24, 0], 2, dtype=dtype)
    for i, keep in ((0, [0, 1, 2, 4, 5, 6]), (1, [1, 2])):
        good.table_np[i, 0, :] = -1
        good.table_np[i, 0, : len(keep)] = c.table_np[i, 0, keep]
    good.pages, good.scales = c.pages, c.scales
    want, want_lse, _, e_out, e_lse, _ = reference(good, q)
    assert bool(((out.double() - want).abs() <= e_out).all())
    assert bool((lse[2] == -math.inf).all()) and bool(((lse.double() - want_lse).abs() <= e_lse)[:2].all())
    assert torch.equal(c.scores[0, :, 48:64], before[0, :, 48:64]) and torch.equal(c.scores[2], before[2])
    bits = c.bits()
    row = q[:, :2].contiguous()
    kv.append(row, row)                                              # sequence 2's newest slot has no page: dropped
    kv.append_decode(row, row, q)
    torch.cuda.synchronize()
    after = c.bits()
    changed = sum(int((a != b).any(dim=-1).sum()) for a, b in zip(bits[:2], after[:2]))
    assert changed <= 2 * 2 * 2                                      # the newest slots of sequences 0 and 1


def test_lengths_outside_the_table_are_cut():
    c = Paged([64, 32], 2)
    c.lengths.copy_(torch.tensor([1 << 30, -5], dtype=torch.int32))
    q = new_q(c, 1)
    out, lse = c.kv.decode_attn(q, return_lse=True)
    assert c.kv.device_status() == 2
    c.n[0], c.n[1] = 64, 0
    want, _, _, e_out, _, _ = reference(c, q)
    assert bool(((out.double() - want).abs() <= e_out).all())


def test_short_score_rows():
    c = Paged([100], 2)
    scores = torch.zeros((1, 2, 60), device="cuda")
    kv = B.PagedKV(c.pages[0], c.pages[1], c.table, c.lengths, scores=scores)
    q = new_q(c, 2)
    kv.decode_attn(q, accumulate=True)
    assert kv.device_status() == 4
    _, _, w, _, _, e = reference(c, q)
    assert bool(((scores.double() - w[..., :60]).abs() <= e[..., :60] + 3 * U * w[..., :60]).all())


# ------------------------------------------------------------------------------------------------ append
def quantized(x):
    x = x.float()
    top = x.abs().amax(dim=-1)
    s = top / torch.full_like(top, 448.0)                            # by a plain number torch would multiply by its inverse
    by = torch.where(s > 0, s, torch.ones_like(s))
    return (x / by[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn), s


def expect_append(c, k_new, v_new, cu):
    """The pages, scales and scores after the rows went in, written one slot at a time."""
    pages = [p.clone() for p in c.pages]
    scales = [None if s is None else s.clone() for s in c.scales]
    scores = None if c.scores is None else c.scores.clone()
    for i in range(c.n.shape[0]):
        for t in range(cu[i], cu[i + 1]):
            for h in range(c.heads):
                slot = int(c.n[i, h]) - (cu[i + 1] - t)
                if slot < 0:
                    continue
                pg, r, hh = int(c.table_np[i, h % c.table_np.shape[1], slot // c.page]), slot % c.page, h % c.pages[0].shape[1]
                for w, new in enumerate((k_new, v_new)):
                    if c.dtype == "e4m3":
                        code, s = quantized(new[t, h])
                        pages[w].view(torch.uint8)[pg, hh, r] = code.view(torch.uint8)
                        scales[w][pg, hh, r] = s
                    else:
                        pages[w][pg, hh, r] = new[t, h]
                if scores is not None:
                    scores[i, h, slot] = 0
    return pages, scales, scores


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def assert_cache(c, want):
    pages, scales, scores = want
    assert all(same_bits(a, b) for a, b in zip(c.pages, pages))
    assert all(a is None or same_bits(a, b) for a, b in zip(c.scales, scales))
    assert scores is None or same_bits(c.scores, scores)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,heads,order,per_head", [(128, 4, "head", False), (64, 5, "token", False), (128, 3, "head", True), (64, 7, "head", True), (128, 1, "token", False)])
def test_append(dtype, d, heads, order, per_head):
    n = np.random.RandomState(d + heads).randint(1, 80, size=(6, heads)) if per_head else np.array([1, 16, 17, 40, 33, 64])
    tokens = np.array([1, 3, 0, 40, 7, 1])
    if per_head:
        tokens = np.minimum(tokens, n.min(axis=1))
    c = Paged(n, heads, d=d, dtype=dtype, order=order, per_head=per_head, scores=True)
    g = torch.Generator(device="cuda").manual_seed(4)
    t = TYPES[dtype if dtype != "e4m3" else "fp16"]
    cu = np.concatenate([[0], np.cumsum(tokens)])
    new = [torch.randn((cu[-1], heads, d), generator=g, device="cuda").to(t) for _ in range(2)]
    new[0][0] = 0                                                    # a row of zeros has a scale of zero
    want = expect_append(c, new[0], new[1], cu)
    c.kv.append(new[0], new[1], torch.from_numpy(cu.astype(np.int32)).cuda())
    assert_cache(c, want)
    # one token per sequence, from a slice of a projection
    both = torch.randn((6, 3 * heads, d), generator=g, device="cuda").to(t)
    k, v = both[:, heads:2 * heads], both[:, 2 * heads:]
    want = expect_append(c, k, v, np.arange(7))
    c.kv.append(k, v)
    assert_cache(c, want)
    assert c.kv.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_rows_of_any_size(dtype, d):
    """Scales and codes are correctly rounded quotients over the whole range of the types, zero, denormal and border values
    included."""
    n_rows = 20000
    g = torch.Generator(device="cuda").manual_seed(d)
    t = TYPES[dtype]
    span = 60 if dtype == "bf16" else 12
    x = torch.randn((n_rows, 1, d), generator=g, device="cuda") * torch.exp2(torch.randint(-2 * span, span, (n_rows, 1, 1), generator=g, device="cuda").float())
    x[::3] *= torch.exp2(torch.randint(-12, 1, x[::3].shape, generator=g, device="cuda").float())
    x[::7] = torch.round(x[::7] * 16) / 16                           # halves between codes, exactly
    x[5], x[6] = 0.0, torch.finfo(t).max
    x[7], x[8, 0, 3:] = torch.finfo(t).smallest_normal / 4, 0.0
    x = x.clamp(-torch.finfo(t).max, torch.finfo(t).max).to(t)
    c = Paged([n_rows], 1, d=d, dtype="e4m3", page=64)
    c.kv.append(x, x, torch.tensor([0, n_rows], dtype=torch.int32, device="cuda"))
    code, scale = quantized(x)
    got = [torch.from_numpy(np.arange(n_rows)).cuda()]
    at = (torch.from_numpy(c.table_np[0, 0].astype(np.int64)).cuda()[got[0] // 64], 0, got[0] % 64)
    for w in range(2):
        assert torch.equal(c.scales[w][at], scale[:, 0])
        bad = (c.pages[w].view(torch.uint8)[at] != code[:, 0].view(torch.uint8)).nonzero()
        assert len(bad) == 0, [(r, i, float(x[r, 0, i]), float(scale[r, 0])) for r, i in bad[:5].tolist()]
    if dtype == "bf16" and d == 128:                                 # and the slab cache's quantiser says the same
        codes, scales = B.quantize_rows_e4m3(x[:, 0].contiguous())
        assert torch.equal(codes, code[:, 0].view(torch.uint8)) and torch.equal(scales, scale[:, 0])


def test_append_for_many_sequences():
    r = np.random.RandomState(1)
    tokens = r.randint(0, 4, size=2500) * r.randint(0, 2, size=2500)
    n = tokens + r.randint(0, 5, size=2500)
    c = Paged(n, 2, d=64, page=8, scores=True)
    cu = np.concatenate([[0], np.cumsum(tokens)])
    new = torch.randn((int(cu[-1]), 2, 64), generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").to(torch.bfloat16)
    seq = np.repeat(np.arange(2500), tokens)
    slot = n[seq] - tokens[seq] + (np.arange(len(seq)) - cu[seq])
    page = torch.from_numpy(c.table_np[seq, 0, slot // 8].astype(np.int64)).cuda()
    at = torch.from_numpy(slot % 8).cuda()
    pages, scores = [p.clone() for p in c.pages], c.scores.clone()
    for p in pages:
        p[page, :, at] = new
    scores[torch.from_numpy(seq).cuda(), :, torch.from_numpy(slot).cuda()] = 0
    c.kv.append(new, new, torch.from_numpy(cu.astype(np.int32)).cuda())
    assert_cache(c, (pages, c.scales, scores))
    c.kv.append(new[:0], new[:0], torch.zeros(2501, dtype=torch.int32, device="cuda"))       # no new tokens at all
    assert_cache(c, (pages, c.scales, scores))
    assert c.kv.device_status() == 0


def test_append_of_more_than_fits():
    c = Paged([5, 20], 2, scores=True)
    cu = np.array([0, 9, 12])
    new = torch.randn((12, 2, 128), device="cuda").to(torch.bfloat16)
    want = expect_append(c, new, new, cu)
    c.kv.append(new, new, torch.from_numpy(cu.astype(np.int32)).cuda())
    assert_cache(c, want)
    assert c.kv.device_status() == 2


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,g,per_head,n_seqs", [(128, 1, False, 14), (64, 4, False, 14), (128, 16, True, 5), (64, 20, True, 6), (128, 2, False, 200)])
def test_append_decode_is_append_then_attention(dtype, d, g, per_head, n_seqs):
    r = np.random.RandomState(n_seqs)
    n = r.randint(0, 150, size=(n_seqs, 3)) if per_head else np.resize(EDGE, n_seqs)
    made = [Paged(n, 3, d=d, dtype=dtype, per_head=per_head, scores=True, page=24) for _ in range(3)]
    q = new_q(made[0], g)
    both = torch.randn((n_seqs, 6, d), device="cuda").to(q.dtype)
    k, v = both[:, :3], both[:, 3:]
    a, b, c = made
    out, lse = a.kv.append_decode(k, v, q, return_lse=True, accumulate=True)
    b.kv.append(k, v)
    before = b.scores.clone()
    out2, lse2 = b.kv.decode_attn(q, return_lse=True, accumulate=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert_cache(a, (b.pages, b.scales, b.scores))
    check_attention(b, q, out2, lse2, before=before)
    out3 = c.kv.append_decode(k, v, q)                               # without the weights: the new slot starts at zero
    assert torch.equal(out3, out) and same_bits(c.scores, before)


# ------------------------------------------------------------------------------------------------ eviction
def expect_evict(c, prefix, budget, recent):
    """Source slots per head."""
    kept = []
    sc = c.scores.cpu().numpy()
    for i in range(c.n.shape[0]):
        row = []
        for h in range(c.heads):
            n = int(c.n[i, h])
            keep = prefix + budget[h] + recent[h]
            if n <= keep:
                row.append(list(range(n)))
                continue
            cand = np.arange(prefix, n - recent[h])
            x = sc[i, h, cand].astype(np.float64)
            x = np.where(np.isnan(x), -np.inf, x)                    # and below -inf, see the key
            nan = np.isnan(sc[i, h, cand])
            best = cand[np.lexsort((cand, nan, -x))][: budget[h]]
            row.append(list(range(prefix)) + sorted(best.tolist()) + list(range(n - recent[h], n)))
        kept.append(row)
    return kept


def check_evict(c, prefix, budget, recent, into=None):
    b = [budget] * c.heads if np.ndim(budget) == 0 else list(budget)
    r = [recent] * c.heads if np.ndim(recent) == 0 else list(recent)
    want = expect_evict(c, prefix, b, r)
    before = [p.clone() for p in c.pages], [None if s is None else s.clone() for s in c.scales], c.scores.clone(), c.lengths.clone()
    to = into or c
    pages = [p.clone() for p in to.pages]
    scales = [None if s is None else s.clone() for s in to.scales]
    scores = None if to.scores is None else to.scores.clone()
    raw = lambda x: x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x  # noqa: E731
    for i, row in enumerate(want):
        for h, src in enumerate(row):
            if not src:
                continue
            s, j = np.asarray(src), np.arange(len(src))
            at = (torch.from_numpy(c.table_np[i, h % c.table_np.shape[1]][s // c.page].astype(np.int64)).cuda(), h % c.pages[0].shape[1],
                  torch.from_numpy(s % c.page).cuda())
            put = (torch.from_numpy(to.table_np[i, h % to.table_np.shape[1]][j // to.page].astype(np.int64)).cuda(), h % to.pages[0].shape[1],
                   torch.from_numpy(j % to.page).cuda())
            for w in range(2):
                raw(pages[w])[put] = raw(before[0][w])[at]
                if scales[w] is not None:
                    scales[w][put] = before[1][w][at]
            if scores is not None:
                scores[i, h, : len(src)] = before[2][i, h, torch.from_numpy(s).cuda()]
    kept = c.kv.evict(prefix, budget, recent, into=None if into is None else into.kv).cpu().numpy()
    for i, row in enumerate(want):
        for h, src in enumerate(row):
            assert kept[i, h, : len(src)].tolist() == src, (i, h)
            assert (kept[i, h, len(src):] == -1).all()
    counts = np.array([[len(x) for x in row] for row in want])
    got = to.lengths.cpu().numpy()
    assert np.array_equal(np.broadcast_to(got[:, None], counts.shape) if got.ndim == 1 else got, counts)
    assert_cache(to, (pages, scales, scores))
    if into is not None:                                             # the source is as it was
        assert_cache(c, before[:3])
        assert torch.equal(c.lengths, before[3])
    assert c.kv.device_status() == 0 and to.kv.device_status() == 0
    to.n = counts
    return counts


def targets(c, seed=9, page=None, order="head", scores=True, top=None):
    n = np.full(c.n.shape, c.max_pages * c.page if top is None else top)
    t = Paged(n, c.heads, d=c.d, dtype=c.dtype, page=page or c.page, order=order, scores=scores, seed=seed)
    return t


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("d,page,order,per_head", [(128, 16, "head", False), (64, 24, "token", False), (128, 7, "head", True), (64, 16, "token", True)])
@pytest.mark.parametrize("place", ["in place", "elsewhere"])
def test_evict(dtype, d, page, order, per_head, place):
    r = np.random.RandomState(page)
    heads = 4
    n = r.randint(0, 400, size=(12, heads))
    n[0], n[1], n[2] = 0, 1, 78                                      # nothing, one, exactly what is kept
    c = Paged(n, heads, d=d, dtype=dtype, page=page, order=order, per_head=per_head, scores=True)
    into = None if place == "in place" else targets(c, page=20, order="token" if order == "head" else "head", top=90)
    check_evict(c, 10, [60, 0, 7, 1], [8, 68, 0, 77], into)


@pytest.mark.parametrize("place", ["in place", "elsewhere"])
def test_evict_ties_zeros_and_nan(place):
    n = np.full((8, 3), 300)
    c = Paged(n, 3, scores=True)
    r = np.random.RandomState(0)
    x = r.randint(0, 6, size=c.scores.shape).astype(np.float32)
    x[1] = 0.0
    x[2] = np.where(r.rand(*x[2].shape) < 0.5, -0.0, 0.0)            # the two zeros are equal
    x[3] = np.nan
    x[4] = np.where(r.rand(*x[4].shape) < 0.9, np.nan, x[4])
    x[5] = np.where(r.rand(*x[5].shape) < 0.3, np.inf, -x[5])
    x[6] = np.where(r.rand(*x[6].shape) < 0.5, -np.inf, 1e-42)       # denormal numbers are not zeros
    c.scores.copy_(torch.from_numpy(x))
    check_evict(c, 5, [100, 20, 1], [10, 0, 30], None if place == "in place" else targets(c, top=120))


@pytest.mark.parametrize("n", [8100, 9000, 60000])
@pytest.mark.parametrize("place", ["in place", "elsewhere"])
def test_evict_long_rows(n, place):
    """Keys in shared memory for 256 and for 1024 threads, and more of them than fit there."""
    c = Paged(np.array([[n, n - 5000], [n - 3, 77]]), 2, d=64, scores=True, page=64)
    c.scores[0, 0] = torch.round(c.scores[0, 0] * 8) / 8             # many equal values
    check_evict(c, 3, [4000, 2500], [64, 1], None if place == "in place" else targets(c, top=4100))


@pytest.mark.parametrize("heads,cap", [(1, 1100), (3, 5000), (2, 40000), (9, 33000), (20, 9000), (40, 6000), (80, 3000), (80, 40000), (3, 100000), (1, 300000), (9, 300000)])
def test_evict_choice_over_many_thread_blocks(heads, cap):
    """The list of long tables alone: one to eight thread blocks per head, keys that fit in shared memory and that do not,
    ties inside a thread block's run and across several, runs without any candidate."""
    r = np.random.RandomState(heads + cap)
    x = np.exp(2.0 * r.randn(heads, cap)).astype(np.float32)
    n = r.randint(cap // 2, cap + 1, size=heads)
    n[0] = cap
    budget, recent = r.randint(1, cap // 3, size=heads), r.randint(0, 40, size=heads)
    for h in range(heads):
        kind = (h + (cap == 300000)) % 9
        if kind == 1:
            x[h] = r.randint(0, 4, size=cap)                         # ties everywhere
        elif kind == 2:
            x[h] = 0.25                                              # nothing else
        elif kind == 3:
            x[h] = 1.0 + r.randint(0, 3000, size=cap) * 2.0 ** -23   # bins of many keys
        elif kind == 4:
            x[h, : cap // 2] = 7.0                                   # the ties in the first thread blocks
        elif kind == 5:
            x[h, cap // 3:] = 1e6                                    # and in the last
        elif kind == 6:
            x[h] = np.where(r.rand(cap) < 0.98, np.nan, x[h])
        elif kind == 7:
            n[h], recent[h] = min(cap, int(budget[h]) + 5 + 3 + 37), 37         # a few more than are kept
        elif kind == 8:
            x[h] = np.where(r.rand(cap) < 0.5, -x[h], x[h])
    page = 64
    one = torch.zeros((1, 1, page, 64), dtype=torch.bfloat16, device="cuda")     # every slot is in the same page
    most = int(3 + (budget + recent).max())
    wide = -(-most // page)
    pool = torch.zeros((heads * wide, 1, page, 64), dtype=torch.bfloat16, device="cuda")
    c = B.PagedKV(one, one.clone(), torch.zeros((1, heads, -(-cap // page)), dtype=torch.int32, device="cuda"),
                  torch.from_numpy(n.astype(np.int32)).cuda()[None], scores=torch.from_numpy(x).cuda()[None])
    to = B.PagedKV(pool, pool.clone(), torch.arange(heads * wide, dtype=torch.int32, device="cuda").view(1, heads, wide),
                   torch.full((1, heads), -1, dtype=torch.int32, device="cuda"), scores=torch.full((1, heads, most), -5.0, device="cuda"))
    kept = c.evict(3, budget.tolist(), recent.tolist(), into=to)[0].cpu().numpy()
    moved, lens = to.scores[0].cpu().numpy(), to.lengths[0].cpu().numpy()
    for h in range(heads):
        k = int(budget[h] + recent[h] + 3)
        if n[h] <= k:
            want = np.arange(n[h])
        else:
            key = x[h, 3:n[h] - recent[h]].astype(np.float64)
            order = np.argsort(-np.where(np.isnan(key), -np.inf, key), kind="stable")[: budget[h]]
            want = np.concatenate([np.arange(3), 3 + np.sort(order), np.arange(n[h] - recent[h], n[h])])
        assert np.array_equal(kept[h, : len(want)], want), h
        assert (kept[h, len(want):] == -1).all() and lens[h] == len(want)
        assert np.array_equal(moved[h, : len(want)], x[h, want], equal_nan=True)
        assert (moved[h, len(want):] == -5.0).all()
    assert c.device_status() == 0 and to.device_status() == 0


def test_evict_again_and_again():
    """One token appended and one evicted, many times over (the recent slots move down by one each time)."""
    c = Paged(np.full((3, 4), 41), 4, scores=True, room=2)
    q = new_q(c, 2)
    for step in range(20):
        check_evict(c, 4, [20, 0, 5, 36], [16, 36, 31, 0])
        assert (c.n == 40).all()
        c.lengths.add_(1)
        c.n = c.n + 1
        new = torch.randn((3, 4, 128), device="cuda").to(torch.bfloat16)
        before = None
        out, lse = c.kv.append_decode(new, new, q, return_lse=True, accumulate=True)
        want, want_lse, _, e_out, e_lse, _ = reference(c, q)
        assert bool(((out.double() - want).abs() <= e_out).all()) and bool(((lse.double() - want_lse).abs() <= e_lse).all())


def test_evict_with_one_length_per_sequence():
    c = Paged(np.array([100, 40, 0, 64]), 4, scores=True)
    check_evict(c, 8, [40, 30, 20, 10], [10, 20, 30, 40])            # the same number of slots for every head
    assert c.lengths.tolist() == [58, 40, 0, 58]
    with pytest.raises(B.SsdError):
        c.kv.evict(8, [40, 30, 20, 11], [10, 20, 30, 40])
    with pytest.raises(B.SsdError):
        c.kv.evict(8, 10, 10, into=c.kv)
    with pytest.raises(ValueError):
        c.kv.evict(8, [1, 2], 10)
    small = targets(c, top=20)
    with pytest.raises(B.SsdError):
        c.kv.evict(8, 30, 10, into=small.kv)


def test_evict_without_scores_at_the_target():
    c = Paged(np.array([[50, 60]]), 2, scores=True)
    check_evict(c, 1, 10, 5, targets(c, top=20, scores=False))


# ------------------------------------------------------------------------------------------------ as it is used
def test_captured_step_follows_lengths_and_pages():
    """One captured decode step (append, attention with weights), replayed while lengths and tables grow."""
    c = Paged([20, 3, 0, 60], 4, scores=True, room=40)
    # the table holds the pages of the rows to come; lengths are advanced by the step itself
    c.n = c.n.copy()
    q, new = new_q(c, 2), torch.randn((4, 8, 128), device="cuda").to(torch.bfloat16)
    k, v = new[:, :4], new[:, 4:]
    out = torch.empty_like(q)
    c.kv.reserve(8, accumulate=True)
    lone = Paged([20, 3, 0, 60], 4, scores=True, room=40)            # the same cache, driven eagerly
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.lengths.add_(1)
        c.kv.append_decode(k, v, q, out=out, accumulate=True)
    for step in range(5):
        q.copy_(new_q(c, 2, seed=step + 20))
        new.copy_(torch.randn(new.shape, device="cuda"))
        g.replay()
        lone.lengths.add_(1)
        want = lone.kv.append_decode(k, v, q, accumulate=True)
        assert torch.equal(out, want) and torch.equal(c.lengths, lone.lengths)
    assert_cache(c, (lone.pages, lone.scales, lone.scores))
    c.n += 5
    want, _, _, e_out, _, _ = reference(c, q)
    assert bool(((out.double() - want).abs() <= e_out).all())


@pytest.mark.parametrize("cap", [64, 2048, 36000])
def test_captured_refresh(cap):
    """Append, attention with weights and eviction in one captured graph, replayed: the same bits as the calls one by one."""
    made = [Paged([50, 20, 0, 61], 4, dtype="e4m3", scores=True, room=cap - 61) for _ in range(2)]
    q, new = new_q(made[0], 2), torch.randn((4, 4, 128), device="cuda").to(torch.bfloat16)
    for c in made:
        c.kv.reserve(8, accumulate=True)
        c.heads_len = torch.from_numpy(np.repeat(c.n[:, :1], 4, 1).astype(np.int32)).cuda()
        c.kv = B.PagedKV(c.pages[0], c.pages[1], c.table, c.heads_len, k_scales=c.scales[0], v_scales=c.scales[1], scores=c.scores)
        c.kv.reserve(8, accumulate=True)
    a, b = made
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.heads_len.add_((a.heads_len > 0).int())
        out = a.kv.append_decode(new, new, q, accumulate=True)
        kept = a.kv.evict(4, [20, 30, 0, 5], [10, 8, 40, 30])
    for step in range(4):
        q.copy_(new_q(b, 2, seed=step + 50))
        new.copy_(torch.randn(new.shape, device="cuda"))
        g.replay()
        b.heads_len.add_((b.heads_len > 0).int())
        want = b.kv.append_decode(new, new, q, accumulate=True)
        want_kept = b.kv.evict(4, [20, 30, 0, 5], [10, 8, 40, 30])
        assert torch.equal(out, want) and torch.equal(kept, want_kept) and torch.equal(a.heads_len, b.heads_len)
        assert_cache(a, (b.pages, b.scales, b.scores))
    assert b.kv.device_status() == 0 and b.heads_len.max().item() <= 44


def test_capture_needs_a_reserved_workspace():
    c = Paged([20], 2)
    q = new_q(c, 1)
    with pytest.raises(RuntimeError, match="reserve"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            c.kv.decode_attn(q)
    torch.cuda.synchronize()
    out, lse = c.kv.decode_attn(q, return_lse=True)
    check_attention(c, q, out, lse)


def test_a_captured_call_keeps_the_workspace_it_was_captured_with():
    c = Paged([900, 33, 400], 4, scores=True)
    q, more, h = new_q(c, 2), new_q(c, 2), c.kv
    h.reserve(8)
    small = h.workspace.data_ptr()
    want = h.decode_attn(q).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = h.decode_attn(q)
    h.decode_attn(more, accumulate=True)                     # a larger workspace
    assert h.workspace.data_ptr() != small
    fresh = [torch.full((n,), 0x55, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 20, 1 << 22)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((x == 0x55).all()) for x in fresh)
    with pytest.raises(ValueError, match="workspace"):
        B.PagedKV(h.k_pages, h.v_pages, h.page_table, h.lengths, workspace=torch.zeros(8, device="cuda"))


def test_caches_of_other_shapes_share_a_workspace():
    a, b = Paged([500, 30], 2), Paged([9, 900, 44], 8, d=64, dtype="fp16")
    a.kv.reserve(64)
    b.kv.workspace = a.kv.workspace
    for _ in range(3):
        for c, g in ((a, 20), (b, 2), (a, 1), (b, 4)):
            q = new_q(c, g)
            out, lse = c.kv.decode_attn(q, return_lse=True)
            check_attention(c, q, out, lse)
    assert b.kv.workspace is a.kv.workspace


def test_another_stream():
    c = Paged([300, 70, 5], 4, scores=True)
    q, before = new_q(c, 2), c.scores.clone()
    want = c.kv.decode_attn(q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out, lse = c.kv.decode_attn(q, return_lse=True, accumulate=True)
    s.synchronize()
    assert torch.equal(out, want)
    check_attention(c, q, out, lse, before=before)


def test_handle_refusals():
    c = Paged([30, 4], 4)
    q = new_q(c, 2)
    bad = [q[:1], q[:, :6], q.to(torch.float16), q.float(), q[..., :64], q[0], q.transpose(1, 2).contiguous().transpose(1, 2), q.cpu()]
    launches = B.kernel_launch_count()
    for x in bad:
        with pytest.raises(ValueError):
            c.kv.decode_attn(x)
    with pytest.raises(ValueError):
        c.kv.decode_attn(q, accumulate=True)                         # no scores
    with pytest.raises(ValueError):
        c.kv.evict(1, 1, 1)
    with pytest.raises(ValueError):
        c.kv.decode_attn(q, out=torch.empty_like(q[:1]))
    with pytest.raises(ValueError):
        c.kv.append(q, q)
    with pytest.raises(ValueError):
        c.kv.append(q[:, :4], q[:, :4].contiguous())                 # other strides
    with pytest.raises(ValueError):
        c.kv.append(q[:1, :4], q[:1, :4])
    with pytest.raises(ValueError):
        c.kv.append(q[:, :4], q[:, :4], torch.zeros(3, device="cuda"))
    odd = torch.empty(2 * 8 * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 8, 128)
    with pytest.raises(B.SsdError):
        c.kv.decode_attn(odd)                                        # 8-byte aligned
    assert B.kernel_launch_count() == launches


def test_generation_with_the_papers_head_split():
    """Algorithm 2 with this cache: prompts of different lengths are appended, every step appends and attends with the weights,
    and whenever the buffer is full each head is cut down by its label's policy.  Sequences of the same length as the slab
    cache's are compared with it, the others with plain arithmetic."""
    w = wl.CONFIGS["tiny"]
    heads, L, W, M, R = w.n_heads, 32, w.window, w.sink_budget, w.sink_recent
    labels = np.array([1, 0, 1, 0, 0, 1, 0, 0])
    budget, recent = B.head_budgets(labels, W, M, R)
    buffer = 12
    n0 = np.array([40, 90, 61])
    room = np.array(budget).max() + max(recent) + L + buffer
    c = Paged(np.zeros((3, heads), np.int64), heads, scores=True, room=max(int(room), 90) + buffer)
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda n: torch.randn((n, heads, 128), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    k, v = new(int(n0.sum())), new(int(n0.sum()))
    c.lengths.copy_(torch.from_numpy(np.repeat(n0[:, None], heads, 1)))
    c.n = np.repeat(n0[:, None], heads, 1)
    cu = np.concatenate([[0], np.cumsum(n0)])
    c.kv.append(k, v, torch.from_numpy(cu.astype(np.int32)).cuda())
    # plain copies of what every head holds, in float64: rows and scores
    held = [[(k[cu[i]:cu[i + 1], h].double(), v[cu[i]:cu[i + 1], h].double(), torch.zeros(n0[i], dtype=torch.float64, device="cuda"))
             for h in range(heads)] for i in range(3)]
    for step in range(30):
        q = (1.5 * torch.randn((3, 2 * heads, 128), generator=g, device="cuda")).to(torch.bfloat16)
        kt, vt = new(3), new(3)
        c.lengths.add_(1)
        c.n = c.n + 1
        out, lse = c.kv.append_decode(kt, vt, q, return_lse=True, accumulate=True)
        _, _, _, e_out, _, _ = reference(c, q)
        for i in range(3):
            for h in range(heads):
                a, b, s = held[i][h]
                a, b = torch.cat([a, kt[i, h].double()[None]]), torch.cat([b, vt[i, h].double()[None]])
                p = torch.softmax(q[i, 2 * h:2 * h + 2].double() @ a.T / math.sqrt(128), dim=1)
                assert bool(((out[i, 2 * h:2 * h + 2].double() - p @ b).abs() <= e_out[i, 2 * h:2 * h + 2]).all())
                held[i][h] = (a, b, torch.cat([s, s.new_zeros(1)]) + p.sum(dim=0))
        if (step + 1) % buffer == 0:
            kept = c.kv.evict(L, budget, recent).cpu().numpy()
            c.n = c.lengths.cpu().numpy().astype(np.int64)
            for i in range(3):
                for h in range(heads):
                    a, b, s = held[i][h]
                    src = torch.from_numpy(kept[i, h][kept[i, h] >= 0].astype(np.int64)).cuda()
                    # the set is the best one up to ties within the scores' own error
                    keep = L + budget[h] + recent[h]
                    assert len(src) == min(len(s), keep)
                    if len(s) > keep and budget[h]:
                        cand = torch.arange(L, len(s) - recent[h], device="cuda")
                        inside = torch.isin(cand, src)
                        assert float(s[cand][~inside].max()) <= float(s[cand][inside].min()) * (1 + 1e-3)
                    held[i][h] = (a[src], b[src], s[src])
                    assert torch.allclose(c.scores[i, h, : len(src)].double(), s[src], rtol=1e-3, atol=1e-6)
    assert c.kv.device_status() == 0


def test_same_result_as_the_slab_cache():
    """One layer of the slab cache in row-buffer mode and this cache with the same rows: the same sets and outputs."""
    w = wl.CONFIGS["tiny"]
    L, N, n0, M, R, H = w.prompt_len, w.n_img, w.n0, w.sink_budget, w.sink_recent, w.n_heads
    cfg = B.make_config(1, 2, H, L, N, w.window, M, R)
    slab = B.SsdCache(cfg)
    slab.set_head_labels(np.ones(H, np.uint8))
    slab.set_row_buffer(True)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((2, H, L + N, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    slab.compress(0, q[:, :, L:L + n0].contiguous(), k[:, :, : L + n0].contiguous(), v[:, :, : L + n0].contiguous(), n0)
    start = slab.get_compress_scores(0, n0)
    c = Paged(np.full((2, H), L + n0), H, scores=True, room=R)
    rows = [x[:, :, : L + n0].permute(0, 2, 1, 3).reshape(-1, H, 128) for x in (k, v)]
    c.kv.append(rows[0], rows[1], torch.tensor([0, L + n0, 2 * (L + n0)], dtype=torch.int32, device="cuda"))
    c.scores[:, :, L:L + n0].copy_(torch.from_numpy(start))
    ids = np.tile(np.arange(L + n0), (2, H, 1))                      # what lies in each slot
    take = lambda kept: np.take_along_axis(ids, np.maximum(kept, 0).astype(np.int64), 2)  # noqa: E731
    ids = take(c.kv.evict(L, M, 0).cpu().numpy())
    assert [set(x) for x in ids.reshape(2 * H, -1)] == [set(x[x >= 0]) for x in slab.get_indices(0).reshape(2 * H, -1)]
    for t in range(n0 + 1, n0 + 1 + 2 * R):
        kt, vt, qt = (x[:, :, L + t - 1].contiguous() for x in (k, v, q))
        c.lengths.add_(1)
        a = slab.append_decode(0, kt, vt, qt)
        b = c.kv.append_decode(kt, vt, qt, accumulate=True)
        ids = np.concatenate([ids, np.full((2, H, 1), L + t - 1)], axis=2)
        # both are within half a step and the arithmetic's error of the exact value: twice that apart at most
        assert float((a.float() - b.float()).abs().max()) <= 2 * (2.0 ** -9 * float(a.float().abs().max()) + 2e-3)
        if (t - n0) % R == 0:
            slab.recompress(0)
            ids = take(c.kv.evict(L, M, 0).cpu().numpy())
            assert [set(x) for x in ids.reshape(2 * H, -1)] == [set(x[x >= 0]) for x in slab.get_indices(0).reshape(2 * H, -1)]
    slab.close()
