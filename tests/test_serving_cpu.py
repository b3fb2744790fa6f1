"""Serving operators without a GPU: what the C calls refuse, and the plain forms the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2203_17189_b200 import binding as Bd
from paper_2203_17189_b200 import build as builder
from tests import serving_reference as SR

P = 1 << 20      # an aligned address that no refused call may touch
NULL, CONFIG, SHAPE, ALIGN, WORKSPACE, ARG = -1, -2, -3, -4, -5, -8


@pytest.fixture(scope="module", autouse=True)
def built():
    builder.build()


APPEND = dict(dtype=1, n_tokens=4, n_heads=4, n_kv_heads=2, d_kv=64, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, q_out=P,
              ldqo=256, seq=P, pos=P, rot_dim=64, rot_base=1e4, inter=0, k_pages=P, v_pages=P, n_pages=8, page=16,
              page_stride=2048, slot_stride=128, head_stride=64, table=P, n_seqs=2, max_pages=4, ld_table=4, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), ARG), (dict(n_tokens=-1), ARG), (dict(d_kv=48), ARG), (dict(n_kv_heads=0), ARG), (dict(n_heads=0), ARG),
    (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(seq=None), NULL),
    (dict(pos=None), NULL), (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(table=None), NULL),
    (dict(rot_dim=-16), ARG), (dict(rot_dim=24), ARG), (dict(rot_dim=80), ARG), (dict(rot_base=0.0), ARG),
    (dict(rot_base=float("nan")), ARG), (dict(inter=2), ARG), (dict(ldq=255), ARG), (dict(ldk=127), ARG), (dict(ldv=64), ARG),
    (dict(ldqo=8), ARG), (dict(ldk=132), ALIGN), (dict(ldq=260), ALIGN), (dict(k=P + 2), ALIGN), (dict(q_out=P + 8), ALIGN),
    (dict(k_pages=P + 8), ALIGN), (dict(slot_stride=130), ALIGN), (dict(head_stride=32), ARG), (dict(page_stride=0), ARG),
    (dict(n_pages=0), ARG), (dict(page=0), ARG), (dict(n_seqs=0), ARG), (dict(max_pages=0), ARG), (dict(ld_table=3), ARG),
    (dict(max_pages=1 << 20, ld_table=1 << 20, page=1 << 11), SHAPE)])
def test_append_refuses(change, code):
    assert Bd.lib().t5_paged_kv_append(*dict(APPEND, **change).values()) == code


def test_append_of_nothing_is_done_on_the_host():
    assert Bd.lib().t5_paged_kv_append(*dict(APPEND, n_tokens=0, k=None, v=None, seq=None, pos=None, q=None,
                                             q_out=None).values()) == 0


ATTEND = dict(dtype=1, n_rows=4, n_q=2, n_heads=4, n_kv_heads=2, d_kv=64, scale=1.0, q=P, ldq=256, k_pages=P, v_pages=P,
              n_pages=8, page=16, page_stride=2048, slot_stride=128, head_stride=64, table=P, max_pages=4, ld_table=4, lens=P,
              bias=P, n_bias=32, out=P, ldo=256, lse=P, ws=P, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), ARG), (dict(n_rows=-2), ARG), (dict(n_rows=3), ARG), (dict(n_q=0), ARG), (dict(n_q=65, n_rows=65), ARG),
    (dict(n_kv_heads=3), ARG), (dict(n_heads=0), ARG), (dict(d_kv=96), ARG), (dict(scale=float("inf")), ARG),
    (dict(scale=float("nan")), ARG), (dict(bias=None), ARG), (dict(n_bias=0), ARG), (dict(n_bias=-1), ARG),
    (dict(q=None), NULL), (dict(k_pages=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL),
    (dict(ws=None), NULL), (dict(ldq=255), ARG), (dict(ldo=128), ARG), (dict(ldq=258), ALIGN), (dict(out=P + 2), ALIGN),
    (dict(q=P + 4), ALIGN), (dict(ws=P + 8), ALIGN), (dict(page_stride=2050), ALIGN), (dict(v_pages=P + 2), ALIGN),
    (dict(ws_bytes=100), WORKSPACE), (dict(max_pages=1 << 20, ld_table=1 << 20, page=1 << 11), SHAPE),
    (dict(n_rows=1 << 22, n_heads=4096, n_kv_heads=4096, n_q=1), SHAPE), (dict(n_pages=0), ARG)])
def test_attention_refuses(change, code):
    assert Bd.lib().t5_paged_attention(*dict(ATTEND, **change).values()) == code


def test_attention_workspace():
    n = C.c_int64()
    assert Bd.lib().t5_paged_attention_workspace_bytes(4, 2, 4, 2, 64, None) == NULL
    assert Bd.lib().t5_paged_attention_workspace_bytes(4, 3, 4, 2, 64, C.byref(n)) == ARG
    sizes = [Bd.t5_paged_attention_workspace_bytes(8, 1, h, 1, 128) for h in (1, 4, 16, 64)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    # it does not grow with the batch or the cache
    assert Bd.t5_paged_attention_workspace_bytes(4096, 1, 4, 1, 128) == sizes[1]
    assert Bd.lib().t5_paged_attention(*dict(ATTEND, n_rows=0, q=None, lens=None, out=None, ws=None).values()) == 0


VERIFY = dict(dtype=0, n_seqs=2, max_draft=3, vocab=100, target=P, ts=400, tr=100, draft=P, ds=300, dr=100, x=P, ldx=3, n=P,
              u=P, ldu=3, us=P, out=P, ldo=4, acc=P, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), ARG), (dict(n_seqs=-1), ARG), (dict(max_draft=-1), ARG), (dict(max_draft=1025, ldx=1025, ldu=1025, ldo=1026), ARG),
    (dict(vocab=0), ARG), (dict(vocab=(1 << 20) + 1, tr=1 << 21, dr=1 << 21), SHAPE), (dict(target=None), NULL), (dict(x=None), NULL),
    (dict(u=None), NULL), (dict(us=None), NULL), (dict(out=None), NULL), (dict(acc=None), NULL), (dict(tr=99), ARG),
    (dict(dr=99), ARG), (dict(ts=-1), ARG), (dict(ldx=2), ARG), (dict(ldu=2), ARG), (dict(ldo=3), ARG), (dict(target=P + 2), ALIGN),
    (dict(draft=P + 1), ALIGN)])
def test_verify_refuses(change, code):
    assert Bd.lib().t5_verify_draft(*dict(VERIFY, **change).values()) == code


def test_plain_attention_is_softmax():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(n, h, 32, generator=g) for n, h in ((1, 4), (24, 2), (24, 2)))
    table = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    out, lse, _, _ = SR.attention(q, k.view(3, 8, 2, 32), v.view(3, 8, 2, 32), table, [21], 8, 1, 0.3, None)
    for h in range(4):
        z = (k[:21, h // 2].double() @ q[0, h].double()) * 0.3
        torch.testing.assert_close(out[0, h], torch.softmax(z, 0) @ v[:21, h // 2].double())
        torch.testing.assert_close(lse[0, h], torch.logsumexp(z, 0))


def test_plain_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 64))
    pos = [0, 5, 100000]
    y = SR.rotate(x, pos, 32, 1e4, True)
    z = (x[..., 0:32:2] + 1j * x[..., 1:32:2]) * np.exp(1j * np.outer(pos, 1e4 ** (-np.arange(16) / 16)))[:, None]
    np.testing.assert_allclose(y[..., 0:32:2], z.real, atol=1e-12)
    np.testing.assert_allclose(y[..., 1:32:2], z.imag, atol=1e-12)
    np.testing.assert_array_equal(y[..., 32:], x[..., 32:])


def test_plain_verification_follows_the_target():
    """Over many random numbers the first token's distribution is the target's, whatever the draft."""
    rng = np.random.default_rng(1)
    p, q = np.array([0.5, 0.3, 0.2, 0.0]), np.array([0.1, 0.2, 0.3, 0.4])
    n = 20000
    x = rng.choice(4, size=(n, 1), p=q)
    target = np.broadcast_to(np.stack([p, p]), (n, 2, 4))
    draft = np.broadcast_to(q[None], (n, 1, 4))
    out, _ = SR.verify(target, draft, x, None, rng.random((n, 1)), rng.random(n))
    seen = np.bincount(out[:, 0], minlength=4) / n
    # five standard deviations of a share over n draws
    assert np.all(np.abs(seen - p) <= 5 * np.sqrt(np.maximum(p * (1 - p), 1e-9) / n))
