"""t5_paged_attention against the plain float64 form, at the lengths, layouts and masks where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_2203_17189_b200 import binding as Bd
from tests import serving_reference as SR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def i32(a):
    return torch.as_tensor(np.asarray(a, dtype=np.int32)).to(DEV)


def build(rng, seq_lens, n_q, h, g, d, page, dtype, layout="slots", n_bias=0, cap=None, spread=1.0):
    """Random caches; every slot behind a sequence's length, and every page of nobody, holds NaN."""
    kp, vp, table = SR.make_pools(rng, [max(cap or 0, n, 1) for n in seq_lens], page, g, d, dtype, DEV, layout)
    gen = torch.Generator(device=DEV).manual_seed(int(rng.integers(1 << 30)))
    for s, n in enumerate(seq_lens):
        pg, sl = SR.slots_of(table, s, n, page)
        kp[pg, sl] = torch.randn(n, g, d, generator=gen, device=DEV).to(dtype)
        vp[pg, sl] = (torch.randn(n, g, d, generator=gen, device=DEV) + 0.5).to(dtype)
    q = (spread * torch.randn(len(seq_lens) * n_q, h, d, generator=gen, device=DEV)).to(dtype)
    lens = [max(n - (n_q - 1 - i), 0) for n in seq_lens for i in range(n_q)]
    bias = torch.randn(h, n_bias, generator=gen, device=DEV) if n_bias else None
    return q, kp, vp, table, lens, bias


def workspace(r, n_q, h, g, d):
    ws = torch.empty(Bd.t5_paged_attention_workspace_bytes(r, n_q, h, g, d), dtype=torch.uint8, device=DEV)
    ws.fill_(0xff)      # NaN patterns: nothing may be read that was not written
    return ws


def widened(table, page):
    """The same pages in a table that could name 2^18 keys: the call may no longer assume a short cache."""
    wide = torch.full((table.shape[0], max(table.shape[1], (1 << 18) // page)), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    return wide


def attend(q, kp, vp, table, lens, scale, n_q, bias, ws=None):
    out = torch.full_like(q, float("nan"), memory_format=torch.contiguous_format)
    lse = torch.full(q.shape[:2], float("nan"), device=DEV)
    ws = workspace(q.shape[0], n_q, q.shape[1], kp.shape[2], q.shape[2]) if ws is None else ws
    Bd.t5_paged_attention(q, kp, vp, table, i32(lens), out, ws, scale=scale, n_q=n_q, bias=bias, lse=lse)
    return out, lse


def check(q, kp, vp, table, lens, scale, n_q, bias):
    out, lse = attend(q, kp, vp, table, lens, scale, n_q, bias)
    ref, rlse, tol, ltol = SR.attention(q, kp, vp, table, lens, kp.shape[1], n_q, scale, bias)
    assert torch.isfinite(out).all()
    off = (out.double() - ref).abs()
    assert bool((off <= tol).all()), f"off by {float((off - tol).max())} over the tolerance at {int((off - tol).argmax())}"
    empty = torch.isinf(rlse)
    assert torch.equal(torch.isinf(lse), empty) and bool((lse[empty] < 0).all())
    loff = (lse.double() - rlse)[~empty].abs()
    assert bool((loff <= ltol[~empty]).all())
    return out, lse


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("seq_lens,n_q,h,g,d,page,n_bias,layout", [
    ([1], 1, 1, 1, 32, 16, 0, "slots"),
    ([1, 0, 2, 15, 16, 17], 1, 4, 4, 32, 16, 8, "slots"),
    ([31, 32, 33, 63, 64, 65, 0, 127, 128, 129], 1, 6, 6, 64, 16, 32, "heads"),
    ([114], 1, 32, 32, 64, 16, 128, "slots"),
    ([255, 256, 257, 511, 513], 1, 8, 2, 64, 24, 128, "mixed"),
    ([1000, 3, 777], 1, 16, 1, 128, 100, 0, "heads"),
    ([2500], 1, 2, 2, 128, 64, 1, "slots"),
    ([9000, 1], 1, 8, 1, 128, 32, 128, "heads"),
    ([20, 5, 4, 1, 0], 5, 4, 4, 64, 7, 128, "slots"),
    ([700, 64, 129], 5, 8, 2, 128, 24, 64, "mixed"),
    ([90, 300], 8, 12, 2, 32, 1, 0, "slots"),
    ([150], 64, 2, 2, 64, 16, 20, "slots"),
    ([70, 333], 1, 40, 2, 64, 16, 0, "heads"),
    ([50, 61], 3, 64, 2, 128, 128, 500, "slots"),
    ([400, 0, 33, 1100], 5, 12, 3, 64, 16, 128, "slots"),
    ([700, 129], 8, 8, 2, 128, 24, 0, "heads"),
    ([90, 257, 64], 17, 2, 2, 64, 16, 40, "mixed"),
    ([310, 20], 16, 9, 3, 32, 16, 64, "slots")])
def test_matches_plain_form(dtype, seq_lens, n_q, h, g, d, page, n_bias, layout, wide):
    rng = np.random.default_rng(len(seq_lens) * 100 + h)
    q, kp, vp, table, lens, bias = build(rng, seq_lens, n_q, h, g, d, page, dtype, layout, n_bias)
    check(q, kp, vp, widened(table, page) if wide else table, lens, d ** -0.5, n_q, bias)


@pytest.mark.parametrize("n_q,h,g,d", [(17, 1, 1, 64), (5, 32, 4, 128), (8, 16, 4, 128), (3, 24, 4, 64), (11, 6, 1, 64), (8, 8, 1, 64),
                                       (64, 2, 1, 128), (64, 3, 1, 64), (9, 15, 1, 128), (33, 4, 4, 128), (20, 2, 2, 32)])
@pytest.mark.parametrize("seq_lens,page,n_bias,layout", [([300, 0, 64, 65, 1000, 1], 16, 32, "slots"), ([5001], 24, 0, "heads"),
                                                         ([63, 129, 128, 0, 0, 2, 700] * 6, 100, 500, "mixed"),
                                                         ([200, 17], 1, 1, "slots")])
def test_many_rows_per_kv_head(n_q, h, g, d, seq_lens, page, n_bias, layout):
    rng = np.random.default_rng(23)
    q, kp, vp, table, lens, bias = build(rng, seq_lens, n_q, h, g, d, page, BF16, layout=layout, n_bias=n_bias)
    table = widened(table, page)
    check(q, kp, vp, table, lens, 0.125, n_q, bias)
    lens = rng.integers(-1, max(seq_lens) + 1, len(lens)).tolist()      # rows of a sequence in no order, some empty
    lens = [min(n, seq_lens[i // n_q]) for i, n in enumerate(lens)]
    check(q, kp, vp, table, lens, 0.125, n_q, bias)


def test_many_rows_agree_bit_for_bit_and_replay_from_a_graph():
    rng = np.random.default_rng(24)
    q, kp, vp, table, lens, bias = build(rng, [9000, 200, 0, 77], 5, 16, 2, 128, 16, BF16, n_bias=128)
    table = widened(table, 16)
    ws = workspace(20, 5, 16, 2, 128)
    first, lse = attend(q, kp, vp, table, lens, 0.1, 5, bias, ws)
    out, lens_d = torch.empty_like(q), i32(lens)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        Bd.t5_paged_attention(q, kp, vp, table, lens_d, out, ws, scale=0.1, n_q=5, bias=bias)
    for _ in range(20):
        out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out, first)
    q.mul_(0.5)
    graph.replay()
    assert torch.equal(out, attend(q, kp, vp, table, lens, 0.1, 5, bias, ws)[0]) and not torch.equal(out, first)


@pytest.mark.parametrize("n_q,h,g,d", [(5, 16, 2, 128), (8, 8, 2, 64), (20, 8, 1, 128)])
def test_many_rows_of_sharp_and_large_scores(n_q, h, g, d):
    rng = np.random.default_rng(25)
    q, kp, vp, table, lens, _ = build(rng, [700, 129, 64], n_q, h, g, d, 16, BF16, spread=30.0)
    check(q, kp, vp, widened(table, 16), lens, 1.0, n_q, None)


@pytest.mark.parametrize("n_q,h,g,d", [(6, 12, 3, 64), (10, 5, 1, 128), (30, 6, 1, 64)])
def test_many_rows_and_a_bias_that_masks(n_q, h, g, d):
    """The lowest value on every key of a head leaves a uniform mean, -infinity an empty row."""
    rng = np.random.default_rng(26)
    q, kp, vp, table, lens, bias = build(rng, [200, 70, 6], n_q, h, g, d, 16, BF16, n_bias=8)
    bias[1], bias[2] = torch.finfo(F32).min, -float("inf")
    out, lse = attend(q, kp, vp, widened(table, 16), lens, 0.1, n_q, bias)
    ref, rlse, tol, ltol = SR.attention(q, kp, vp, table, lens, 16, n_q, 0.1, bias)
    others = [i for i in range(h) if i not in (1, 2)]
    assert bool(((out.double() - ref).abs() <= tol)[:, others].all())
    assert not out[:, 2].any() and bool((lse[:, 2] == -float("inf")).all())
    for r, n in enumerate(lens):
        pg, sl = SR.slots_of(table, r // n_q, n, 16)
        v = vp[pg, sl][:, 1 // (h // g)].double()
        want = v.mean(0) if n else torch.zeros(d, device=DEV)
        assert (out[r, 1].double() - want).abs().max() <= (SR.HALF[BF16] + 2.0 ** -15) * (v.abs().max() if n else 1)


def test_many_rows_and_pages_that_are_none():
    rng = np.random.default_rng(27)
    n_q, h, g, d = 5, 10, 2, 128
    q, kp, vp, table, _, _ = build(rng, [330], n_q, h, g, d, 24, BF16)
    good, table = table.clone(), widened(table, 24)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    Bd.t5_kernel_status_word(status)
    try:
        attend(q, kp, vp, table, [300] * n_q, 0.1, n_q, None)
        assert status.item() == 0
        table[0, 1], table[0, 6], table[0, 7] = kp.shape[0], -1, -2 ** 31
        out, _ = attend(q, kp, vp, table, [300] * n_q, 0.1, n_q, None)
        assert status.item() == 202
    finally:
        Bd.t5_kernel_status_word(None)
    keep = [j for j in range(300) if j // 24 not in (1, 6, 7)]
    pg, sl = SR.slots_of(good, 0, 300, 24)
    k, v = (x[pg, sl][keep].double().repeat_interleave(h // g, 1) for x in (kp, vp))
    w = torch.softmax(torch.einsum("nhd,rhd->rhn", k, q.double()) * 0.1, -1)
    ref = torch.einsum("rhn,nhd->rhd", w, v)
    assert (out.double() - ref).abs().max() <= (SR.HALF[BF16] + 2.0 ** -12) * v.abs().max()


def test_many_rows_of_a_cache_beyond_four_gigabytes():
    n_pages, page, g, d, n_q = 4200, 64, 64, 128, 20
    kp = torch.empty(n_pages, page, g, d, dtype=BF16, device=DEV)
    vp = torch.empty_like(kp)
    table = i32([[n_pages - 1, 0, n_pages - 2]])
    for p in table[0].tolist():
        kp[p], vp[p] = torch.randn(page, g, d, device=DEV).to(BF16), torch.randn(page, g, d, device=DEV).to(BF16)
    q = torch.randn(n_q, g, d, device=DEV).to(BF16)
    check(q, kp, vp, widened(table, 64), [150 - i for i in range(n_q)], 0.09, n_q, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_sequences_of_every_length(dtype):
    """More sequences than threads look at at once, in no order of length, many of them empty."""
    rng = np.random.default_rng(11)
    seq_lens = rng.integers(0, 90, 700).tolist()
    seq_lens[::5] = [0] * len(seq_lens[::5])
    q, kp, vp, table, lens, bias = build(rng, seq_lens, 1, 3, 3, 64, 16, dtype, n_bias=40)
    check(q, kp, vp, table, lens, 0.2, 1, bias)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lengths_of_a_sequences_rows_in_no_order(dtype, wide):
    """Rows that share a sequence may see any number of its keys, none included."""
    rng = np.random.default_rng(12)
    q, kp, vp, table, _, bias = build(rng, [300, 300, 40], 6, 4, 2, 64, 16, dtype, n_bias=17)
    table = widened(table, 16) if wide else table
    lens = [300, 0, 1, 150, 64, 299, 0, 0, 0, 300, 17, 16, 0, -3, 40, 39, 1, 2]
    check(q, kp, vp, table, lens, 0.125, 6, bias)


@pytest.mark.parametrize("dtype,n_q,h,g", [(F32, 4, 4, 4), (BF16, 4, 4, 4), (BF16, 4, 8, 2), (BF16, 8, 8, 2), (BF16, 11, 4, 2), (BF16, 20, 6, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("wide", [False, True])
def test_keys_a_row_does_not_see_may_hold_anything(dtype, n_q, h, g, bad, wide):
    """The later tokens of a draft hold NaN or infinities: the earlier rows do not notice."""
    rng = np.random.default_rng(13)
    q, kp, vp, table, lens, bias = build(rng, [100, 67], n_q, h, g, 64, 16, dtype, n_bias=128)
    table = widened(table, 16) if wide else table
    want, want_lse = attend(q, kp, vp, table, lens, 0.1, n_q, bias)
    for s, n in enumerate([100, 67]):
        pg, sl = SR.slots_of(table, s, n, 16)
        kp[pg[-1], sl[-1]] = bad
        vp[pg[-1], sl[-1]] = bad
    out, lse = attend(q, kp, vp, table, lens, 0.1, n_q, bias)
    earlier = torch.arange(2 * n_q) % n_q != n_q - 1
    assert torch.isfinite(out[earlier]).all()
    ref, rlse, tol, ltol = SR.attention(q, kp, vp, table, lens, 16, n_q, 0.1, bias)
    assert bool(((out[earlier].double() - ref[earlier]).abs() <= tol[earlier]).all())
    assert bool(((lse[earlier].double() - rlse[earlier]).abs() <= ltol[earlier]).all())
    # both calls are roundings of the same exact values
    assert bool(((out[earlier].double() - want[earlier].double()).abs() <= 2 * tol[earlier]).all())
    # and the row that does see it is spoilt in every column, as the formula says
    if bad != bad:
        assert torch.isnan(out[~earlier]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low", [-float("inf"), torch.finfo(F32).min])
@pytest.mark.parametrize("wide", [False, True])
def test_bias_that_masks(dtype, low, wide):
    """A bias of the type's lowest value or of -infinity: on the far keys it removes them; on all keys the lowest value
    leaves a uniform mean, -infinity an empty row."""
    rng = np.random.default_rng(14)
    q, kp, vp, table, lens, bias = build(rng, [200, 33, 5], 1, 2, 2, 64, 16, dtype, n_bias=64)
    table = widened(table, 16) if wide else table
    bias[0, :40] = low      # head 0 sees the nearest 24 keys
    bias[1] = low           # head 1 sees nothing, or everything alike
    out, lse = attend(q, kp, vp, table, lens, 0.1, 1, bias)
    for r, n in enumerate(lens):
        pg, sl = SR.slots_of(table, r, n, 16)
        k, v = kp[pg, sl].double(), vp[pg, sl].double()
        near = slice(max(n - 24, 0), n)
        z = k[near, 0] @ q[r, 0].double() * 0.1 + bias[0, 64 - min(n, 24):].double()
        want = torch.softmax(z, 0) @ v[near, 0]
        scale = float(v.abs().max())
        # scores of about 3 (10 roundings of 2^-24 of them), 200 terms, one rounding to the output type
        tol = (SR.HALF[dtype] + 2.0 ** -15) * scale
        assert (out[r, 0].double() - want).abs().max() <= tol
        if low == -float("inf"):
            assert not out[r, 1].any() and lse[r, 1] == -float("inf")
        else:
            assert (out[r, 1].double() - v[:, 1].mean(0)).abs().max() <= tol
            assert torch.isfinite(lse[r, 1])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sharp_and_large_scores(dtype, wide):
    """Scores of several hundred: the maximum moves often, the rest underflows to nothing."""
    rng = np.random.default_rng(15)
    q, kp, vp, table, lens, bias = build(rng, [400, 129], 1, 4, 2, 128, 16, dtype, spread=30.0)
    table = widened(table, 16) if wide else table
    check(q, kp, vp, table, lens, 1.0, 1, None)


def test_strided_rows_and_shared_pages():
    rng = np.random.default_rng(16)
    h, g, d, page = 4, 2, 64, 16
    _, kp, vp, table, _, _ = build(rng, [96], 1, h, g, d, page, BF16)
    # three sequences share the first pages (a common prompt); wide tables and wide rows
    wide = torch.full((3, 20), -1, dtype=torch.int32, device=DEV)
    wide[:, :6] = table[0]
    big = torch.randn(3, (h + 3) * d, device=DEV).to(BF16)
    q = big[:, d:(h + 1) * d].view(3, h, d)
    out_big = torch.full((3, h * d + 64), float("nan"), dtype=BF16, device=DEV)
    out = out_big[:, :h * d].view(3, h, d)
    lens = [96, 40, 0]
    ws = workspace(3, 1, h, g, d)
    Bd.t5_paged_attention(q, kp, vp, wide[:, :6], i32(lens), out, ws, scale=0.125)
    ref, _, tol, _ = SR.attention(q, kp, vp, wide, lens, page, 1, 0.125, None)
    assert bool(((out.double() - ref).abs() <= tol).all())
    assert torch.isnan(out_big[:, h * d:]).all()


def test_cache_beyond_four_gigabytes():
    """Offsets that pass 32 bits, in bytes and in elements."""
    rng = np.random.default_rng(17)
    n_pages, page, g, d = 4200, 64, 64, 128
    kp = torch.empty(n_pages, page, g, d, dtype=BF16, device=DEV)
    vp = torch.empty_like(kp)
    table = i32([[n_pages - 1, 0, n_pages - 2]])
    for p in table[0].tolist():
        kp[p], vp[p] = torch.randn(page, g, d, device=DEV).to(BF16), torch.randn(page, g, d, device=DEV).to(BF16)
    q = torch.randn(1, g, d, device=DEV).to(BF16)
    check(q, kp, vp, table, [150], 0.09, 1, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wide", [False, True])
def test_bad_pages_and_lengths_are_reported(wide, dtype):
    rng = np.random.default_rng(18)
    q, kp, vp, table, lens, _ = build(rng, [64, 64], 1, 2, 2, 64, 16, dtype)
    table = widened(table, 16) if wide else table
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    Bd.t5_kernel_status_word(status)
    try:
        good = table.clone()
        want, _ = attend(q, kp, vp, good, [64, 64], 0.1, 1, None)
        assert status.item() == 0
        table[0, 1], table[1, 3] = kp.shape[0], -1
        out, _ = attend(q, kp, vp, table, [64, 64], 0.1, 1, None)
        assert status.item() == 202
        # the keys of a bad page count as absent
        for r, keep in ((0, [0, 2, 3]), (1, [0, 1, 2])):
            pg = good[r, keep].long()
            k, v = kp[pg].reshape(-1, 2, 64).double(), vp[pg].reshape(-1, 2, 64).double()
            w = torch.softmax(torch.einsum("nhd,hd->hn", k, q[r].double()) * 0.1, -1)
            ref = torch.einsum("hn,nhd->hd", w, v)
            assert (out[r].double() - ref).abs().max() <= (SR.HALF[dtype] + 2.0 ** -12) * v.abs().max()
        status.zero_()
        if not wide:      # a length beyond what the table can name is cut to that
            out, _ = attend(q, kp, vp, good, [64, 1000], 0.1, 1, None)
            assert status.item() == 203 and torch.equal(out, want)
        else:             # here it reaches into entries that name no page
            out, _ = attend(q, kp, vp, good, [64, 1000], 0.1, 1, None)
            assert status.item() == 202 and torch.isfinite(out).all()
            status.zero_()
            attend(q, kp, vp, good, [64, (1 << 18) + 1], 0.1, 1, None)
            assert status.item() in (202, 203)
    finally:
        Bd.t5_kernel_status_word(None)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_runs_agree_bit_for_bit_and_replay_from_a_graph(dtype):
    rng = np.random.default_rng(19)
    q, kp, vp, table, lens, bias = build(rng, [5000, 200, 0, 77], 1, 8, 4, 64, 16, dtype, n_bias=128)
    h, g, d = 8, 4, 64
    ws = workspace(4, 1, h, g, d)
    first, lse = attend(q, kp, vp, table, lens, 0.1, 1, bias, ws)
    second, _ = attend(q, kp, vp, table, lens, 0.1, 1, bias)
    assert torch.equal(first, second)
    dl, out = i32(lens), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        Bd.t5_paged_attention(q, kp, vp, table, dl, out, ws, scale=0.1, bias=bias)
        with torch.cuda.graph(graph, stream=side):
            Bd.t5_paged_attention(q, kp, vp, table, dl, out, ws, scale=0.1, bias=bias)
            Bd.t5_paged_attention(q, kp, vp, table, dl, out, ws, scale=0.1, bias=bias)
    torch.cuda.current_stream().wait_stream(side)
    for change in (lens, [1, 200, 33, 0], [5000, 1, 1, 1]):
        if change[2]:
            pg, sl = SR.slots_of(table, 2, 33, 16)
            kp[pg, sl], vp[pg, sl] = torch.randn(33, g, d, device=DEV).to(dtype), torch.randn(33, g, d, device=DEV).to(dtype)
        dl.copy_(i32(change))
        out.fill_(float("nan"))
        graph.replay()
        graph.replay()
        want, _ = attend(q, kp, vp, table, change, 0.1, 1, bias)
        assert torch.equal(out, want)


def test_two_streams_with_a_workspace_each():
    rng = np.random.default_rng(20)
    a = build(rng, [4000, 100], 1, 8, 2, 128, 16, BF16)
    b = build(rng, [50, 3000], 1, 8, 2, 128, 16, BF16)
    want = [attend(*x[:5], 0.1, 1, None)[0] for x in (a, b)]
    lens = [i32(x[4]) for x in (a, b)]
    outs = [torch.empty_like(x[0]) for x in (a, b)]
    wss = [workspace(2, 1, 8, 2, 128) for _ in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, s, o, ws, ln in zip((a, b), streams, outs, wss, lens):
            with torch.cuda.stream(s):
                Bd.t5_paged_attention(x[0], x[1], x[2], x[3], ln, o, ws, scale=0.1)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_empty_batch_and_output_over_the_queries():
    rng = np.random.default_rng(22)
    q, kp, vp, table, lens, _ = build(rng, [300, 41], 1, 4, 2, 64, 16, BF16)
    ws = workspace(2, 1, 4, 2, 64)
    Bd.t5_paged_attention(q[:0], kp, vp, table[:0], i32([]), q[:0], ws)
    for wide in (table, widened(table, 16)):
        want, _ = attend(q, kp, vp, wide, lens, 0.1, 1, None, ws)
        over = q.clone()
        Bd.t5_paged_attention(over, kp, vp, wide, i32(lens), over, ws, scale=0.1)
        assert torch.equal(over, want)


def test_binding_refuses_wrong_tensors():
    rng = np.random.default_rng(21)
    q, kp, vp, table, lens, bias = build(rng, [30, 30], 1, 4, 2, 64, 16, BF16, n_bias=8)
    out, ws, ln = torch.empty_like(q), workspace(2, 1, 4, 2, 64), i32(lens)
    for args, kw, code in [((q.float(), kp, vp, table, ln, out, ws), {}, -8), ((q, kp, vp, table, ln, out[:1], ws), {}, -8),
                           ((q, kp, vp, table, ln[:1], out, ws), {}, -8), ((q, kp, vp, table, ln.long(), out, ws), {}, -8),
                           ((q, kp, vp, table[:1], ln, out, ws), {}, -8), ((q, kp, vp, table, ln, out, ws), dict(n_q=2), -8),
                           ((q, kp, vp, table, ln, out, ws), dict(bias=bias.bfloat16()), -8),
                           ((q, kp, vp, table, ln, out, ws), dict(bias=bias[:2]), -8), ((q, kp, vp, table, ln, out, ws[:64]), {}, -5),
                           ((q, kp, vp, table, ln, out, ws), dict(lse=torch.empty(2, 5, device=DEV)), -8),
                           ((q[:, :3], kp, vp, table, ln, out[:, :3], ws), {}, -8), ((q, kp[..., :32], vp[..., :32], table, ln, out, ws), {}, -8)]:
        with pytest.raises(Bd.T5Error) as e:
            Bd.t5_paged_attention(*args, **kw)
        assert e.value.code == code
