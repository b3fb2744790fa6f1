"""The model's decoding step over paged caches: sequences at positions of their own, several new tokens at a time, must give
row t of the teacher-forced logits; and the serving calls together - step, verification of drafts, step - must give the
tokens of plain greedy decoding."""
import numpy as np
import pytest
import torch

from paper_2203_17189_b200 import binding as Bd
from paper_2203_17189_b200 import workloads as WL
from tests import parity as PR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def to_dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Model:
    def __init__(self, arch, dtype, d_kv, S, seed=6):
        if arch == 0:
            self.dims = WL.model_dims("small", n_enc_layers=1, n_dec_layers=2, vocab=512, d_model=128, n_heads=2, d_kv=d_kv,
                                      d_ff=256, enc_len=40, dec_len=150, batch=S, padding=0.2)
        else:
            self.dims = WL.model_dims("declm", n_dec_layers=2, vocab=512, d_model=128, n_heads=2, d_kv=d_kv, d_ff=256,
                                      dec_len=150, batch=S, packed=False)
        self.arch, self.S, self.V = arch, S, 512
        self.Te, self.T = (self.dims["enc_len"] if arch == 0 else 0), self.dims["dec_len"]
        self.h = Bd.Handle(Bd.make_config(self.dims, S, max(self.Te, 1), self.T, dtype))
        man, n = self.h.t5_param_manifest(), self.h.t5_param_count()
        named = WL.make_params(PR.oracle_shapes_from_manifest(man), seed, stddev=0.05, scale_jitter=0.05)
        self.params = torch.from_numpy(PR.pack_params(man, n, named)).to(DEV).to(self.h.torch_dtype)
        self.batch = WL.make_batch(self.dims, seed=5)
        self.dev_batch = {k: to_dev(v) for k, v in self.batch.items()}
        self.ws = torch.empty(self.h.t5_workspace_bytes(), dtype=torch.uint8, device=DEV)
        self.enc_out = self.cross = None
        if arch == 0:
            self.enc_out = torch.empty(S, self.Te, 128, dtype=self.h.torch_dtype, device=DEV)
            self.h.t5_encode(self.params, self.dev_batch, self.enc_out, self.ws)
            self.cross = torch.empty(self.h.t5_decode_cache_bytes(S, self.Te, 1), dtype=torch.uint8, device=DEV)
            self.h.t5_decode_begin(self.params, S, self.Te, 1, self.dev_batch["enc_tokens"], self.enc_out, self.cross)

    def pages(self, page, rng):
        per = -(-self.T // page)
        self.n_pages, self.page = self.S * per + 2, page
        table = rng.permutation(self.n_pages)[:self.S * per].reshape(self.S, per).astype(np.int32)
        self.table = to_dev(table)
        self.pool = torch.full((self.h.t5_decode_pool_bytes(self.n_pages, page),), 0xff, dtype=torch.uint8, device=DEV)

    def step(self, tokens, positions):
        """[S, n] numpy -> logits [S, n, V]"""
        S, n = tokens.shape
        logits = torch.empty(S, n, self.V, dtype=self.h.torch_dtype, device=DEV)
        ws = torch.full((self.h.t5_decode_step_paged_workspace_bytes(S, n),), 0xff, dtype=torch.uint8, device=DEV)
        self.h.t5_decode_step_paged(self.params, self.pool, self.n_pages, self.page, self.table, to_dev(tokens.astype(np.int32)),
                                    to_dev(positions.astype(np.int32)), logits, ws, self.cross, self.Te)
        self.h.t5_device_status(ws)
        return logits


@pytest.mark.parametrize("arch,dtype,d_kv,page", [(0, "f32", 32, 16), (0, "bf16", 64, 24), (1, "bf16", 64, 16), (1, "bf16", 128, 64),
                                                  (1, "f32", 32, 1), (0, "bf16", 32, 8)])
def test_steps_at_positions_of_their_own_reproduce_teacher_forced_logits(arch, dtype, d_kv, page):
    S = 4
    rng = np.random.default_rng(page)
    m = Model(arch, dtype, d_kv, S)
    m.pages(page, rng)
    tgt = m.batch["dec_targets"].copy()
    full = torch.empty(S, m.T, m.V, dtype=m.h.torch_dtype, device=DEV)
    m.h.t5_decode_logits(m.params, m.dev_batch, m.enc_out, full, m.ws)
    ref = full.float().cpu().numpy()
    dec_in = np.zeros_like(tgt)
    dec_in[:, 1:] = tgt[:, :-1]
    valid = tgt != 0
    # as in the cached decoding of rectangular batches: float32 to 1e-4, bfloat16 to 2e-2 of the largest logit
    tol = (1e-4 if dtype == "f32" else 2e-2) * np.abs(ref).max()
    end = valid.sum(1)
    at = np.zeros(S, dtype=np.int64)
    done = np.zeros_like(valid)
    for n in [1, 1, 16, 1, 5, 64, 1, 3, 40, 64, 64]:
        tokens, positions = np.zeros((S, n), np.int64), np.full((S, n), -1, np.int64)
        for s in range(S):
            take = min(n if rng.random() < 0.8 else int(rng.integers(0, n + 1)), int(end[s] - at[s]))
            tokens[s, :take] = dec_in[s, at[s]:at[s] + take]
            positions[s, :take] = np.arange(at[s], at[s] + take)
        # a wrong draft first: its keys and values must be gone when the positions are written again
        m.step(np.where(positions >= 0, (tokens + 7) % 512, 0), positions)
        got = m.step(tokens, positions).float().cpu().numpy()
        for s in range(S):
            for i in range(n):
                if positions[s, i] >= 0:
                    p = positions[s, i]
                    assert np.abs(got[s, i] - ref[s, p]).max() <= tol, (s, p, n)
                    done[s, p] = True
            at[s] = max(at[s], positions[s].max() + 1)
    assert done.sum() >= 0.9 * valid.sum()


@pytest.mark.parametrize("arch,dtype,n_draft", [(1, "f32", 4), (0, "f32", 3), (1, "f32", 6)])
def test_verified_drafts_give_the_tokens_of_greedy_decoding(arch, dtype, n_draft):
    """Greedy target probabilities (one at the largest logit): whatever the drafts are, the emitted tokens are those of
    one-by-one decoding.  Drafts: the right token three times in four.  (float32: in bfloat16 two logits may be equal.)"""
    S, steps = 3, 40
    rng = np.random.default_rng(3)
    m = Model(arch, dtype, 64, S)
    m.pages(16, rng)
    # one by one
    want = np.zeros((S, steps + n_draft + 1), np.int64)
    tok = np.zeros((S, 1), np.int64)
    for t in range(want.shape[1]):
        best = m.step(tok, np.full((S, 1), t)).float().argmax(-1).cpu().numpy()
        want[:, t] = best[:, 0]
        tok = best
    # drafts
    m.pool.fill_(0xff)
    got = [[] for _ in range(S)]
    last, at, calls = np.zeros(S, np.int64), np.zeros(S, np.int64), 0
    out = torch.empty(S, n_draft + 1, dtype=torch.int32, device=DEV)
    acc = torch.empty(S, dtype=torch.int32, device=DEV)
    while min(at) < steps:
        drafts = np.stack([np.where(rng.random(n_draft) < 0.75, want[s, at[s]:at[s] + n_draft], rng.integers(0, 512, n_draft))
                           if at[s] + n_draft < want.shape[1] else np.zeros(n_draft, np.int64) for s in range(S)])
        tokens = np.concatenate([last[:, None], drafts], 1)
        active = at < steps
        positions = np.where(active[:, None], at[:, None] + np.arange(n_draft + 1)[None], -1)
        logits = m.step(np.where(active[:, None], tokens, 0), positions).float()
        probs = torch.nn.functional.one_hot(logits.argmax(-1), 512).float()
        Bd.t5_verify_draft(probs, None, to_dev(drafts.astype(np.int32)), None,
                           to_dev((rng.random((S, n_draft)) * 0.998 + 1e-3).astype(np.float32)),
                           to_dev(rng.random(S).astype(np.float32)), out, acc)
        o, a = out.cpu().numpy(), acc.cpu().numpy()
        for s in range(S):
            if active[s]:
                got[s] += o[s, :a[s] + 1].tolist()
                last[s] = o[s, a[s]]
                at[s] += a[s] + 1
        calls += 1
    for s in range(S):
        assert got[s][:steps] == want[s, :steps].tolist()
    assert calls < steps


def test_a_step_replays_from_a_graph():
    rng = np.random.default_rng(4)
    m = Model(1, "bf16", 64, 2)
    m.pages(16, rng)
    tok, pos = to_dev(np.zeros((2, 1), np.int32)), to_dev(np.zeros((2, 1), np.int32))
    logits = torch.empty(2, 1, 512, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(m.h.t5_decode_step_paged_workspace_bytes(2, 1), dtype=torch.uint8, device=DEV)

    def call():
        m.h.t5_decode_step_paged(m.params, m.pool, m.n_pages, m.page, m.table, tok, pos, logits, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    replayed, plain = [], []
    for where in (replayed, plain):
        m.pool.fill_(0xff)
        for t in range(40):
            tok.copy_(to_dev(np.array([[t % 500], [(3 * t) % 500]], np.int32)))
            pos.fill_(t)
            graph.replay() if where is replayed else call()
            where.append(logits.clone())
    # the row statistics of the folded norms are summed with atomics: equal to a rounding of the operand type
    scale = max(float(x.float().abs().max()) for x in plain)
    for a, b in zip(replayed, plain):
        assert (a.float() - b.float()).abs().max() <= 2e-2 * scale


def test_paged_step_errors():
    m = Model(1, "f32", 32, 2)
    m.pages(16, np.random.default_rng(0))
    ok = dict(n_pages=m.n_pages, page=m.page, pool=m.pool, n=1)

    def call(n_pages, page, pool, n, ws_bytes=None, pos=0):
        tok = torch.zeros(2, n, dtype=torch.int32, device=DEV)
        logits = torch.empty(2, n, 512, device=DEV)
        ws = torch.empty(ws_bytes or m.h.t5_decode_step_paged_workspace_bytes(2, min(n, 64)), dtype=torch.uint8, device=DEV)
        m.h.t5_decode_step_paged(m.params, pool, n_pages, page, m.table, tok, tok + pos, logits, ws)
        m.h.t5_device_status(ws)
    call(**ok)
    for change, code in ((dict(pool=m.pool[:4096]), -5), (dict(ws_bytes=4096), -5), (dict(n=65), -3), (dict(page=0), -3),
                         (dict(n_pages=m.n_pages + 1), -5), (dict(pos=10 ** 6), -3)):
        with pytest.raises(Bd.T5Error) as e:
            call(**{**ok, **change})
        assert e.value.code == code, change
    with pytest.raises(Bd.T5Error):
        m.h.t5_decode_step_paged_workspace_bytes(3, 1)
