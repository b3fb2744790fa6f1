"""t5_verify_draft against the plain float64 form: whole numbers, equal in every case."""
import numpy as np
import pytest
import torch

from paper_2203_17189_b200 import binding as Bd
from tests import serving_reference as SR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a, dtype):
    return None if a is None else torch.as_tensor(np.ascontiguousarray(a)).to(DEV).to(dtype)


def run(target, draft, tokens, n_draft, ua, us):
    """target, draft: device tensors; the rest numpy."""
    s, k1, _ = target.shape
    out = torch.full((s, k1), -9, dtype=torch.int32, device=DEV)
    acc = torch.full((s,), -9, dtype=torch.int32, device=DEV)
    Bd.t5_verify_draft(target, draft, dev(tokens, torch.int32), dev(n_draft, torch.int32), dev(ua, torch.float32),
                       dev(us, torch.float32), out, acc)
    return out.cpu().numpy(), acc.cpu().numpy()


def check(target, draft, tokens, n_draft, ua, us):
    out, acc = run(target, draft, tokens, n_draft, ua, us)
    ref, racc = SR.verify(target.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy(), tokens,
                          n_draft, ua, us)
    np.testing.assert_array_equal(acc, racc)
    np.testing.assert_array_equal(out, ref)
    return out, acc


def inputs(rng, s, k, v, dtype, with_draft):
    z = 2.0 * rng.standard_normal((s, k + 1, v))
    p = np.exp(z) / np.exp(z).sum(-1, keepdims=True)
    y = z[:, :k] + 0.5 * rng.standard_normal((s, k, v))
    q = np.exp(y) / np.exp(y).sum(-1, keepdims=True)
    tokens = np.array([[int(np.searchsorted(np.cumsum(q[i, j]), rng.random() * 0.999)) for j in range(k)] for i in range(s)],
                      dtype=np.int32).reshape(s, k)
    return (dev(p, dtype), dev(q, dtype) if with_draft else None, np.minimum(tokens, v - 1), rng.random((s, k)).astype(np.float32),
            rng.random(s).astype(np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("s,k,v", [(1, 4, 512), (5, 3, 1000), (40, 5, 333), (3, 0, 32128), (2, 8, 32128), (7, 1, 1), (6, 2, 7),
                                   (300, 2, 130), (2, 1, 130001), (2, 40, 64)])
def test_matches_plain_form(dtype, with_draft, s, k, v):
    rng = np.random.default_rng(s * 100 + k)
    target, draft, tokens, ua, us = inputs(rng, s, k, v, dtype, with_draft)
    check(target, draft, tokens, None, ua, us)
    if k:
        n = rng.integers(0, k + 1, s).astype(np.int32)
        n[0] = 0
        check(target, draft, tokens, n, ua, us)


def test_the_largest_vocabulary():
    rng = np.random.default_rng(2)
    v = 1 << 20
    target = torch.rand(1, 2, v, device=DEV)
    draft = torch.rand(1, 1, v, device=DEV)
    for us in (0.0, 0.5, 0.99999994):
        check(target, draft, np.array([[v - 1]], np.int32), None, np.array([[0.999]], np.float32), np.array([us], np.float32))
        check(target, None, np.array([[v - 1]], np.int32), None, np.array([[1e-9]], np.float32), np.array([us], np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_draws_on_a_border(dtype):
    """Uniform probabilities of a power of two and random numbers on the borders between tokens: the sums are exact, the
    first token whose sum lies beyond the border is drawn."""
    v = 4096
    target = torch.full((v, 1, v), 1.0 / v, device=DEV, dtype=dtype)
    out, _ = run(target, None, np.zeros((v, 0), np.int32), None, np.zeros((v, 0), np.float32),
                 (np.arange(v) / v).astype(np.float32))
    np.testing.assert_array_equal(out[:, 0], np.arange(v))


def test_accepting_is_strict_and_exact():
    """u draft < target is decided without rounding."""
    p, q = np.float32(0.3), np.float32(0.7)
    u = np.float32(p / q)
    near = np.array([np.nextafter(u, np.float32(0)), u, np.nextafter(u, np.float32(1)), 0.0], np.float32).reshape(4, 1)
    target = torch.zeros(4, 2, 16, device=DEV)
    draft = torch.zeros(4, 1, 16, device=DEV)
    target[:, 0, 3], draft[:, 0, 3], target[:, 1, 9], target[:, 0, 5] = float(p), float(q), 1.0, 0.7
    _, acc = check(target, draft, np.full((4, 1), 3, np.int32), None, near, np.full(4, 0.4, np.float32))
    np.testing.assert_array_equal(acc, [int(float(x) * float(q) < float(p)) for x in near[:, 0]])


def test_all_accepted_none_accepted_and_equal_distributions():
    rng = np.random.default_rng(4)
    target, draft, tokens, _, us = inputs(rng, 6, 4, 500, torch.float32, True)
    _, acc = check(target, draft, tokens, None, np.zeros((6, 4), np.float32), us)
    assert (acc == 4).all()
    target[np.arange(6), 0, tokens[:, 0]] = 0
    out, acc = check(target, draft, tokens, None, np.zeros((6, 4), np.float32), us)
    assert (acc == 0).all() and (out[:, 1:] == -1).all() and (out[:, 0] >= 0).all()
    same = target[:, :4].clone()
    _, acc = check(target, same, tokens, None, np.full((6, 4), 0.999, np.float32), us)


def test_values_without_mass_and_tokens_out_of_range():
    rng = np.random.default_rng(5)
    target, draft, tokens, ua, us = inputs(rng, 8, 3, 200, torch.float32, True)
    target[0, :, ::3] = float("nan")
    target[1, :, ::2] = float("inf")
    target[2] = -1.0                      # nothing to draw from
    target[3, 0] = draft[3, 0]            # refused below, and nothing is left of the difference
    target[3, 0, 7], draft[3, 0, 7], tokens[3, 0] = 0.0, 0.0, 7
    tokens[4, 0], tokens[5, 1], tokens[6, 0] = -1, 200, 1 << 30
    draft[7, :, ::2] = float("nan")
    out, acc = check(target, draft, tokens, None, ua, us)
    assert out[2, 0] == -1 and acc[3] == 0 and out[3, 0] >= 0 and acc[4] == 0 and acc[6] == 0
    check(target, None, tokens, None, ua, us)


def test_random_numbers_at_the_ends():
    rng = np.random.default_rng(6)
    target, draft, tokens, ua, _ = inputs(rng, 4, 2, 700, torch.float32, True)
    target[:, :, 690:] = 0      # the last tokens with mass lie before the row's end
    check(target, draft, tokens, None, ua, np.array([0.0, 1.0, np.nextafter(np.float32(1), np.float32(0)), 0.0], np.float32))


@pytest.mark.parametrize("s,v", [(3, 5), (3, 700), (3, 32128), (200, 90)])
def test_random_numbers_out_of_range(s, v):
    """Below the range, and NaN: the first token with mass; above it: the last."""
    target = torch.zeros(s, 1, v, device=DEV)
    target[:, 0, 2:v - 1] = 0.25
    us = np.resize(np.array([-0.5, np.nan, 7.0, -np.inf, np.inf, -1e-30], np.float32), s)
    out, acc = run(target, None, np.zeros((s, 0), np.int32), None, np.zeros((s, 0), np.float32), us)
    np.testing.assert_array_equal(out[:, 0], np.where(us > 1, v - 2, 2))
    assert (acc == 0).all()


def test_output_over_the_drafted_tokens():
    rng = np.random.default_rng(10)
    target, draft, tokens, ua, us = inputs(rng, 7, 3, 900, torch.float32, True)
    want, _ = run(target, draft, tokens, None, ua, us)
    over, acc = torch.zeros(7, 4, dtype=torch.int32, device=DEV), torch.empty(7, dtype=torch.int32, device=DEV)
    over[:, :3] = dev(tokens, torch.int32)
    Bd.t5_verify_draft(target, draft, over[:, :3], None, dev(ua, torch.float32), dev(us, torch.float32), over, acc)
    np.testing.assert_array_equal(over.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(dtype):
    """Rows on no 16-byte boundary, and positions outermost."""
    rng = np.random.default_rng(7)
    target, draft, tokens, ua, us = inputs(rng, 5, 3, 301, dtype, True)
    check(target, draft, tokens, None, ua, us)
    want = run(target, draft, tokens, None, ua, us)
    wide = torch.full((5, 4, 320), float("nan"), dtype=dtype, device=DEV)
    wide[..., 3:304] = target
    outer = draft.transpose(0, 1).contiguous().transpose(0, 1)
    got = run(wide[..., 3:304], outer, tokens, None, ua, us)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_graph_replay_and_rows_left_alone():
    rng = np.random.default_rng(8)
    target, draft, tokens, ua, us = inputs(rng, 9, 3, 900, torch.float32, True)
    x, u, w = dev(tokens, torch.int32), dev(ua, torch.float32), dev(us, torch.float32)
    big = torch.full((12, 6), -77, dtype=torch.int32, device=DEV)
    out, acc = big[:9, :4], torch.empty(9, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        Bd.t5_verify_draft(target, draft, x, None, u, w, out, acc)
        with torch.cuda.graph(graph, stream=side):
            Bd.t5_verify_draft(target, draft, x, None, u, w, out, acc)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        ua, us = rng.random((9, 3)).astype(np.float32), rng.random(9).astype(np.float32)
        u.copy_(dev(ua, torch.float32)), w.copy_(dev(us, torch.float32))
        graph.replay()
        ref, racc = SR.verify(target.double().cpu().numpy(), draft.double().cpu().numpy(), tokens, None, ua, us)
        np.testing.assert_array_equal(out.cpu().numpy(), ref)
        np.testing.assert_array_equal(acc.cpu().numpy(), racc)
    assert (big[9:] == -77).all() and (big[:, 4:] == -77).all()


def test_binding_refuses_wrong_tensors():
    rng = np.random.default_rng(9)
    target, draft, tokens, ua, us = inputs(rng, 3, 2, 100, torch.float32, True)
    x, u, w = dev(tokens, torch.int32), dev(ua, torch.float32), dev(us, torch.float32)
    out, acc = torch.empty(3, 3, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    for args in [(target.double(), draft, x, None, u, w, out, acc), (target, draft.bfloat16(), x, None, u, w, out, acc),
                 (target, draft[:, :1], x, None, u, w, out, acc), (target, draft, x.long(), None, u, w, out, acc),
                 (target, draft, x, x[:, 0].float(), u, w, out, acc), (target, draft, x, None, u[:2], w, out, acc),
                 (target, draft, x, None, u, w[:2], out, acc), (target, draft, x, None, u, w, out[:, :2], acc),
                 (target, draft, x, None, u, w, out, acc.long()), (target.transpose(1, 2), draft, x, None, u, w, out, acc)]:
        with pytest.raises(Bd.T5Error) as e:
            Bd.t5_verify_draft(*args)
        assert e.value.code == -8
