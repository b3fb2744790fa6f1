"""t5_paged_kv_append against the plain float64 form: placement exact, rotation to a rounding, nothing else touched."""
import numpy as np
import pytest
import torch

from paper_2203_17189_b200 import binding as Bd
from tests import serving_reference as SR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make_tokens(rng, n, h, g, d, dtype):
    qkv = torch.from_numpy(rng.standard_normal((n, (h + 2 * g) * d)).astype(np.float32)).to(DEV).to(dtype)
    return (qkv[:, :h * d].view(n, h, d), qkv[:, h * d:(h + g) * d].view(n, g, d), qkv[:, (h + g) * d:].view(n, g, d))


def i32(a):
    return torch.as_tensor(np.asarray(a, dtype=np.int32)).to(DEV)


def check(k, v, q, q_out, kp, vp, kp0, vp0, table, seq, pos, page, rot, base, inter):
    real = [i for i, p in enumerate(pos) if p >= 0]
    want_k, want_v = kp0.clone(), vp0.clone()
    t = table.cpu().numpy()
    pg, sl = [int(t[seq[i], pos[i] // page]) for i in real], [pos[i] % page for i in real]
    turned = [max(p, 0) for p in pos]

    def expect(x):
        y = SR.rotate(x.double().cpu().numpy(), turned, rot, base, inter)
        # sine and cosine: 2^-25 turns of the angle and 2 ulp; two products and a sum in float32; the final rounding
        big = np.abs(x.double().cpu().numpy()).max(axis=(1, 2), keepdims=True)
        return y, SR.HALF[x.dtype] * np.abs(y) * (1 + 2.0 ** -7) + 2 * big * (2 * np.pi * 2.0 ** -25 + 5 * 2.0 ** -24) * (rot > 0)

    def compare(got, x, at):
        y, tol = expect(x)
        assert np.all(np.abs(got.double().cpu().numpy() - y[at]) <= tol[at])
        assert torch.equal(got[..., rot:], x[at][..., rot:])

    if real:
        compare(kp[pg, sl], k, real)
        want_k[pg, sl], want_v[pg, sl] = kp[pg, sl], v[real]
    assert torch.equal(torch.nan_to_num(vp, nan=7.0), torch.nan_to_num(want_v, nan=7.0))
    assert torch.equal(torch.nan_to_num(kp, nan=7.0), torch.nan_to_num(want_k, nan=7.0))
    if q is not None:
        compare(q_out, q, list(range(len(pos))))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_seqs,new,h,g,d,page,rot,inter,layout", [
    (1, 1, 1, 1, 32, 16, 0, False, "slots"), (4, 1, 4, 4, 32, 1, 32, False, "slots"), (3, 5, 6, 2, 64, 24, 64, True, "heads"),
    (2, 37, 4, 1, 128, 64, 128, False, "mixed"), (2, 37, 4, 4, 128, 100, 48, True, "heads"), (70, 1, 32, 32, 64, 16, 0, False, "slots"),
    (5, 130, 3, 3, 64, 7, 16, False, "mixed"), (1, 1, 64, 64, 128, 128, 128, True, "slots"), (600, 5, 2, 1, 32, 8, 16, True, "slots")])
def test_append_matches_plain_form(dtype, n_seqs, new, h, g, d, page, rot, inter, layout):
    rng = np.random.default_rng(n_seqs * 1000 + new)
    cap = new + 300
    kp, vp, table = SR.make_pools(rng, [cap] * n_seqs, page, g, d, dtype, DEV, layout)
    kp0, vp0 = kp.clone(), vp.clone()
    q, k, v = make_tokens(rng, n_seqs * new, h, g, d, dtype)
    seq = np.repeat(np.arange(n_seqs), new)
    start = rng.integers(0, cap - new + 1, n_seqs)
    pos = (start[:, None] + np.arange(new)[None]).reshape(-1)
    if new > 8:
        pos[new - 3:new] = -1      # a padded tail
    order = rng.permutation(len(pos))      # tokens in no order
    seq, pos = seq[order], pos[order]
    q_out = torch.full((n_seqs * new, h, d), float("nan"), dtype=dtype, device=DEV)
    Bd.t5_paged_kv_append(k, v, kp, vp, table, i32(seq), i32(pos), q=q, q_out=q_out, rot_dim=rot, rot_base=500.0,
                          rot_interleaved=inter)
    check(k, v, q, q_out, kp, vp, kp0, vp0, table, seq.tolist(), pos.tolist(), page, rot, 500.0, inter)


def test_far_positions_keep_their_angle():
    """Position 10^9: the angle in float32 alone would be off by whole turns."""
    rng = np.random.default_rng(5)
    page, d = 1 << 16, 64
    max_pages = (1 << 30) // page
    kp = torch.zeros(2, page, 1, d, device=DEV)
    vp = torch.zeros_like(kp)
    table = torch.zeros(1, max_pages, dtype=torch.int32, device=DEV)
    table[0, 1000000007 // page] = 1
    q, k, v = make_tokens(rng, 1, 1, 1, d, torch.float32)
    q_out = torch.empty_like(q)
    pos = [1000000007]
    kp0, vp0 = kp.clone(), vp.clone()
    Bd.t5_paged_kv_append(k, v, kp, vp, table, i32([0]), i32(pos), q=q, q_out=q_out, rot_dim=d)
    check(k, v, q, q_out, kp, vp, kp0, vp0, table, [0], pos, page, d, 1e4, False)


def test_queries_rotate_in_place_and_without_queries():
    rng = np.random.default_rng(6)
    kp, vp, table = SR.make_pools(rng, [40, 40], 16, 2, 64, torch.bfloat16, DEV)
    q, k, v = make_tokens(rng, 10, 4, 2, 64, torch.bfloat16)
    seq, pos = i32([0] * 5 + [1] * 5), i32(list(range(5)) + list(range(30, 35)))
    q1, q2 = torch.empty(10, 4, 64, dtype=torch.bfloat16, device=DEV), q.clone()
    Bd.t5_paged_kv_append(k, v, kp, vp, table, seq, pos, q=q, q_out=q1, rot_dim=64)
    k1, v1 = kp.clone(), vp.clone()
    Bd.t5_paged_kv_append(k, v, kp, vp, table, seq, pos, q=q2, q_out=q2, rot_dim=64)
    assert torch.equal(q1, q2)
    kp.fill_(float("nan")), vp.fill_(float("nan"))
    Bd.t5_paged_kv_append(k, v, kp, vp, table, seq, pos, rot_dim=64)
    assert torch.equal(torch.nan_to_num(kp), torch.nan_to_num(k1)) and torch.equal(torch.nan_to_num(vp), torch.nan_to_num(v1))


def test_append_reaches_beyond_four_gigabytes():
    """Offsets that pass 32 bits, in bytes and in elements."""
    rng = np.random.default_rng(7)
    n_pages, page, g, d = 4200, 64, 64, 128      # 2.2e9 elements, 4.4 GB a pool
    kp = torch.empty(n_pages, page, g, d, dtype=torch.bfloat16, device=DEV)
    vp = torch.empty_like(kp)
    kp[-1], vp[-1] = 0, 0
    q, k, v = make_tokens(rng, 2, 1, g, d, torch.bfloat16)
    table = i32([[n_pages - 1]])
    Bd.t5_paged_kv_append(k, v, kp, vp, table, i32([0, 0]), i32([0, 63]))
    assert torch.equal(kp[-1, [0, 63]], k) and torch.equal(vp[-1, [0, 63]], v)
    assert not kp[-1, 1:63].any()


def test_tokens_without_a_place_are_left_out_and_reported():
    rng = np.random.default_rng(8)
    kp, vp, table = SR.make_pools(rng, [32, 32], 16, 1, 32, torch.float32, DEV)
    table[1, 1] = kp.shape[0]      # out of range
    table[0, 1] = -5
    q, k, v = make_tokens(rng, 6, 1, 1, 32, torch.float32)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    Bd.t5_kernel_status_word(status)
    try:
        Bd.t5_paged_kv_append(k, v, kp, vp, table, i32([0, 1, 0, 2, -1, 1]), i32([3, 20, 17, 0, 0, 32]))
        assert status.item() == 201
    finally:
        Bd.t5_kernel_status_word(None)
    assert torch.equal(vp[table[0, 0].long(), 3], v[0])
    assert int((~torch.isnan(kp)).sum()) == 32 and int((~torch.isnan(vp)).sum()) == 32


def test_no_tokens_and_all_padding():
    rng = np.random.default_rng(10)
    kp, vp, table = SR.make_pools(rng, [32], 16, 2, 32, torch.float32, DEV)
    q, k, v = make_tokens(rng, 3, 2, 2, 32, torch.float32)
    Bd.t5_paged_kv_append(k[:0], v[:0], kp, vp, table, i32([]), i32([]), q=q[:0], q_out=q[:0].clone(), rot_dim=32)
    q_out = torch.empty_like(q)
    Bd.t5_paged_kv_append(k, v, kp, vp, table, i32([0, 7, -1]), i32([-1, -5, -2 ** 31]), q=q, q_out=q_out, rot_dim=32)
    assert torch.isnan(kp).all() and torch.isnan(vp).all() and torch.equal(q_out, q)


def test_binding_refuses_wrong_tensors():
    rng = np.random.default_rng(9)
    kp, vp, table = SR.make_pools(rng, [32], 16, 2, 32, torch.float32, DEV)
    q, k, v = make_tokens(rng, 2, 2, 2, 32, torch.float32)
    seq, pos = i32([0, 0]), i32([0, 1])
    for args, kw in [((k.bfloat16(), v, kp, vp, table, seq, pos), {}), ((k, v[:1], kp, vp, table, seq, pos), {}),
                     ((k, v, kp[:, :, :1], vp, table, seq, pos), {}), ((k, v, kp, vp.transpose(0, 1), table, seq, pos), {}),
                     ((k, v, kp, vp, table.long(), seq, pos), {}), ((k, v, kp, vp, table, seq.cpu(), pos), {}),
                     ((k, v, kp, vp, table, seq, pos[:1]), {}), ((k, v, kp, vp, table, seq, pos), dict(q=q)),
                     ((k, v, kp, vp, table, seq, pos), dict(q=q, q_out=q[:1])), ((k, v, kp, vp, table, seq, pos), dict(rot_dim=8)),
                     ((k.transpose(1, 2).contiguous().transpose(1, 2), v, kp, vp, table, seq, pos), {})]:
        with pytest.raises(Bd.T5Error) as e:
            Bd.t5_paged_kv_append(*args, **kw)
        assert e.value.code == -8
