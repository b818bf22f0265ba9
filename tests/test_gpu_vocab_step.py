"""The embedding, verified drafts and distillation used together and with what was there: one
round of generation into the buffer and one training step; graphs, streams, two calls at once,
and tensors whose offsets pass 32 bits."""

import numpy as np
import pytest
import torch

from gpu_util import require_gpu, to_np
from oracle import vocab
from oracle.grad import logprob_backward
from oracle.loss import grpo_loss

pytestmark = pytest.mark.gpu


def _generate(rbp, W, B, K, seed):
    """B sequences of one verified step from a toy policy: (tokens, logp, counts), checked."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    V = W.shape[0]
    hidden = torch.randn((B * (K + 1), W.shape[1]), generator=g, device="cuda").bfloat16()
    logits = (hidden.float() @ W.float().t()).bfloat16().view(B, K + 1, V)
    draft = (logits[:, :K].float()
             + 0.3 * torch.randn((B, K, V), generator=g, device="cuda")).bfloat16()
    pick = torch.rand((B, K, V), generator=g, device="cuda").log_().neg_().log_().neg_()
    x = (draft.float() + pick).argmax(-1).int()
    u = torch.rand((B, K + 1), generator=g, device="cuda")
    tokens = torch.empty((B, K + 1), dtype=torch.int32, device="cuda")
    logp, n = torch.empty((B, K + 1), device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    rbp.policy_verify_drafts(logits, draft, x, None, u, tokens, logp, n,
                             rbp.workspace(rbp.RBP_OP_VERIFY, B, K, V))
    for i in range(0, B, 5):
        want, lp = vocab.verify(to_np(logits[i].double()), to_np(draft[i].double()), to_np(x[i]), K,
                                to_np(u[i]).astype(np.float64))
        assert tokens[i, :len(want)].tolist() == want and n[i].item() == len(want)
        assert np.abs(to_np(logp[i, :len(want)]) - lp).max() < 1e-6 * max(1, np.abs(lp).max())
    return tokens, logp, n


def test_generate_push_draw_embed_distill_and_update():
    rbp = require_gpu()
    V, d, B, K, G = 700, 64, 24, 3, 4
    rng = np.random.default_rng(1)
    W = torch.from_numpy(rng.standard_normal((V, d)) * 0.3).to(torch.bfloat16).cuda()
    # generation: tokens with the behaviour log-probs of the verified steps, pushed as rollouts
    tokens, logp, n = _generate(rbp, W, B, K, 5)
    ring = rbp.make_ring(32, K + 1)
    off = torch.arange(0, B + 1, G, dtype=torch.int32, device="cuda")
    src = torch.arange(B, dtype=torch.int64, device="cuda") * (K + 1)
    reward = torch.from_numpy((rng.random(B) < 0.5).astype(np.float32)).cuda()
    rbp.rb_push(ring, off, n, src, reward, 3, tokens.view(-1), logp.view(-1))
    # a padded batch of it
    cfg = rbp.make_sample_cfg(rbp.RB_UNIFORM, rbp.RB_LAYOUT_PADDED, 7, 0, 16, cur_version=4,
                              l_max=K + 1)
    b = rbp.alloc_batch(cfg)
    rbp.rb_sample_gather(rbp.ring_records(ring), cfg, b,
                         rbp.workspace(rbp.RBP_OP_SAMPLE_GATHER, ring.capacity))
    T = 16 * (K + 1)
    y, seq, length = to_np(b["tokens"]), to_np(b["seq_of_token"]), to_np(b["len"])
    assert (seq < 0).any() and (seq >= 0).any()
    # the trunk is the embedding itself: hidden = 0.5 * W[token]
    hidden = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    rbp.policy_embed_fwd(W, b["tokens"], b["seq_of_token"], hidden, scale=0.5)
    want_h = vocab.embed(to_np(W.double()), y, seq, 0.5)
    assert np.array_equal(to_np(hidden.double()), want_h)  # a power of two: exact
    # the policy gradient on the batch, and the divergence from a teacher beside it
    out = [torch.empty(T, device="cuda") for _ in range(3)]
    dlogp, dhidden = torch.empty(T, device="cuda"), torch.empty((T, d), device="cuda")
    dW = torch.empty((V, d), device="cuda")
    loss, stats = torch.zeros(1, device="cuda"), torch.zeros(4, device="cuda")
    rbp.policy_fused_fwd_bwd(hidden, W, b["tokens"], b["seq_of_token"], b["old_logp"], b["adv"],
                             b["len"], 16, out[0], out[1], out[2], loss, dlogp, stats, dhidden, dW,
                             rbp.workspace(rbp.RBP_OP_FUSED, T, d, V))
    logits = hidden.float() @ W.float().t()
    ids = torch.from_numpy(rng.integers(0, V, (T, 8)).astype(np.int32)).cuda()
    top = torch.from_numpy(rng.standard_normal((T, 8)).astype(np.float32)).cuda()
    kl, dl = torch.empty(T, device="cuda"), torch.empty_like(logits)
    dloss, dstats = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
    rbp.policy_distill_fwd_bwd(logits, ids, top, None, b["seq_of_token"], b["len"], 16, kl, dloss,
                               dstats, dl, rbp.workspace(rbp.RBP_OP_DISTILL, T, 8, V), scale=0.25)
    # both gradients of the hidden states through the embedding, into the tied dW
    dhidden += dl @ W.float()
    dW += dl.t() @ hidden.float()
    rbp.policy_embed_bwd(dhidden, b["tokens"], b["seq_of_token"], dW,
                         rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V), scale=0.5,
                         accumulate_dW=True)
    # the same in fp64
    Wd, h = to_np(W.double()), want_h
    z = h @ Wd.T
    lse = np.log(np.exp(z - z.max(1)[:, None]).sum(1)) + z.max(1)
    valid = seq >= 0
    lp = np.where(valid, z[np.arange(T), np.where(valid, y, 0)] - lse, 0.0)
    wloss, wdlogp, _ = grpo_loss(lp, to_np(b["old_logp"]).astype(np.float64), seq,
                                 to_np(b["adv"]).astype(np.float64), length, 16)
    # each term is a ratio exp(lp - old) of log-probs known to about 4e-6, times its weight
    rho = np.where(valid, np.exp(lp - to_np(b["old_logp"])), 0.0)
    size = (rho * np.abs(to_np(b["adv"]))[np.where(valid, seq, 0)]
            / (16.0 * length[np.where(valid, seq, 0)])).sum()
    assert abs(loss.item() - wloss) < 1e-5 * size + 1e-7
    dh, dw = logprob_backward(h, Wd, y, lse, wdlogp, seq)
    wkl, wdl_loss, _, dz = vocab.distill(to_np(logits.double()), to_np(ids), to_np(top), None, seq,
                                         length, 16, 1.0, 0.25)
    assert abs(dloss.item() - wdl_loss) < 1e-5 * wdl_loss
    dh += dz @ Wd
    dw += dz.T @ h
    want = vocab.embed_backward(dh, y, seq, V, 0.5, dw)
    # (the head's share holds dz in bf16: 2e-3; the rest is fp32)
    assert np.linalg.norm(to_np(dW) - want) < 5e-3 * np.linalg.norm(want)


class Calls:
    """Every new entry point on buffers of its own (and a shared workspace, if given)."""

    def __init__(self, rbp, seed, shared=None):
        self.rbp = rbp
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def f(*shape, sd=1.0):
            return torch.randn(shape, generator=g, device="cuda") * sd

        def i(hi, *shape, lo=0):
            return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)

        T, d, V, B, K = 700, 136, 3001, 9, 3
        self.table, self.tok, self.seq = f(V, d).bfloat16(), i(V, T), i(4, T, lo=-1)
        self.emb, self.dx, self.dW = torch.empty((T, d), device="cuda").bfloat16(), f(T, d), f(V, d)
        self.z, self.zd = f(B, K + 1, V, sd=2).bfloat16(), f(B, K, V, sd=2).bfloat16()
        self.x, self.u = i(V, B, K), torch.rand((B, K + 1), generator=g, device="cuda")
        self.o = [i(2, B, K + 1), f(B, K + 1), i(2, B)]
        self.lg, self.ids, self.lt = f(T, V, sd=2), i(V, T, 16), f(T, 16)
        self.len = torch.full((4,), 30, dtype=torch.int32, device="cuda")
        self.kl, self.loss, self.st = f(T), torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
        self.dl = torch.empty_like(self.lg)
        sizes = [(rbp.RBP_OP_EMBED_BWD, T, d, V), (rbp.RBP_OP_VERIFY, B, K, V),
                 (rbp.RBP_OP_DISTILL, T, 16, V), (rbp.RBP_OP_DISTILL, 2, 16, V * 6)]
        n = max(rbp.rbp_workspace_bytes(*s) for s in sizes)
        self.ws = shared if shared is not None else torch.empty(n, dtype=torch.uint8, device="cuda")
        self.few, self.dfew = f(2, V * 6), torch.empty((2, V * 6), device="cuda")

    def run(self, stream=None):
        r, k = self.rbp, dict(stream=stream)
        r.policy_embed_fwd(self.table, self.tok, self.seq, self.emb, scale=2.0, **k)
        r.policy_verify_drafts(self.z, self.zd, self.x, None, self.u, *self.o, self.ws, **k)
        r.policy_distill_fwd_bwd(self.lg, self.ids, self.lt, None, self.seq, self.len, 4, self.kl,
                                 self.loss, self.st, self.dl, self.ws, **k)
        r.policy_distill_fwd_bwd(self.few, self.ids[:2], self.lt[:2], None, self.seq[:2], self.len, 4,
                                 self.kl[:2], self.loss, self.st, self.dfew, self.ws, **k)
        r.policy_embed_bwd(self.dx, self.tok, self.seq, self.dW, self.ws, **k)
        r.policy_embed_bwd(self.dx, self.tok, self.seq, self.dW, self.ws, accumulate_dW=True, **k)

    def outputs(self):
        return [self.emb, self.kl, self.loss, self.st, self.dl, self.dfew, self.dW, *self.o]

    def eager(self):
        self.reset()
        self.run()
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]

    def reset(self, junk=False):
        self.loss.zero_()
        self.st.zero_()
        if junk:
            for t in (self.emb, self.kl, self.dl, self.dfew, self.dW):
                t.fill_(float("nan"))
            for t in self.o:
                t.fill_(-77)
        torch.cuda.synchronize()


def _equal(got, want):
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graphs_that_share_a_workspace():
    """Two captured sequences of calls on one workspace, replayed in turn with eager calls and
    changed inputs between them."""
    rbp = require_gpu()
    a = Calls(rbp, 1)
    b = Calls(rbp, 2, shared=a.ws)
    graphs = []
    for c in (a, b):
        c.eager()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.run()
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        print("[graph] capture", flush=True)
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    want = [a.eager(), b.eager()]
    for r in range(3):
        for c, g, w in zip((a, b), graphs, want):
            c.reset(junk=True)
            a.ws.fill_(r * 85)
            torch.cuda.synchronize()
            print(f"[graph] replay {r}", flush=True)
            g.replay()
            torch.cuda.synchronize()
            _equal(c.outputs(), w)
        a.u.copy_(1.0 - a.u)
        a.tok.copy_(a.tok.flip(0))
        want[0] = a.eager()


def test_given_streams_and_two_calls_at_once():
    rbp = require_gpu()
    calls = [Calls(rbp, s) for s in (3, 4)]
    want = [c.eager() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for r in range(3):
        for c in calls:
            c.reset(junk=True)
        for c, s in zip(calls, streams):
            c.run(stream=s)
        torch.cuda.synchronize()
        for c, w in zip(calls, want):
            _equal(c.outputs(), w)


def test_the_capturing_stream_is_used():
    """Nothing runs before the replay: every launch was on the current stream."""
    rbp = require_gpu()
    c = Calls(rbp, 6)
    want = c.eager()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    c.reset(junk=True)
    with torch.cuda.graph(g, stream=s):
        c.run()
    torch.cuda.synchronize()
    assert c.dl.isnan().all() and (c.o[0] == -77).all() and c.emb.isnan().all()
    g.replay()
    torch.cuda.synchronize()
    _equal(c.outputs(), want)


def test_logits_beyond_32_bit_offsets():
    rbp = require_gpu()
    V, T, K = 151937, 14500, 4     # 2.2e9 elements
    rng = np.random.default_rng(2)
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    dz = torch.full((T, V), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1, T - 2, T - 1]
    few = torch.from_numpy(rng.standard_normal((4, V))).to(torch.bfloat16)
    seq = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    for k, r in enumerate(rows):
        z[r] = few[k].cuda()
        seq[r] = 0
    ids = torch.from_numpy(rng.integers(0, V, (T, K)).astype(np.int32)).cuda()
    lt = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda()
    length = torch.ones(1, dtype=torch.int32, device="cuda")
    kl, loss, stats = (torch.zeros(n, device="cuda") for n in (T, 1, 2))
    print("[offsets] distill", flush=True)
    rbp.policy_distill_fwd_bwd(z, ids, lt, None, seq, length, 1, kl, loss, stats, dz,
                               rbp.workspace(rbp.RBP_OP_DISTILL, T, K, V))
    wkl, wloss, _, wdz = vocab.distill(to_np(few.double()), to_np(ids[rows]), to_np(lt[rows]), None,
                                       [0] * 4, [1], 1)
    assert stats[0].item() == 4 and np.abs(to_np(kl[rows]) - wkl).max() < 1e-5
    got = to_np(dz[rows].double())
    # half a bf16 step, and what two fp32 terms near each other leave
    assert np.all(np.abs(got - wdz) <= 2.0 ** -8 * np.abs(wdz) + 1e-6)
    assert not dz[2:T - 2].any()
    # the same logits as 3625 sequences of four positions
    B = T // 4
    x = torch.zeros((B, 3), dtype=torch.int32, device="cuda")
    n = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    n[0] = n[B - 1] = 3
    u = torch.full((B, 4), 0.999, device="cuda")
    u[:, 3] = 0.3
    tok = torch.empty((B, 4), dtype=torch.int32, device="cuda")
    lp, cnt = torch.empty((B, 4), device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    print("[offsets] verify", flush=True)
    rbp.policy_verify_drafts(z.view(B, 4, V), z.view(B, 4, V)[:, :3].contiguous(), x, n, u, tok, lp,
                             cnt, rbp.workspace(rbp.RBP_OP_VERIFY, B, 3, V))
    for i in (0, B - 1):
        zi = to_np(z[4 * i:4 * i + 4].double())
        want, wlp = vocab.verify(zi, zi[:3], [0, 0, 0], 3, [0.999, 0.999, 0.999, 0.3])
        # (u beside a step of 1 / 151937 aside, the token is the oracle's)
        assert tok[i, :len(want)].tolist() == want and cnt[i].item() == len(want)
    assert (cnt[1:-1] == 0).all() and (tok[1:-1] == -1).all()


def test_tables_beyond_32_bit_offsets():
    rbp = require_gpu()
    V, d, T = 300007, 8192, 200   # 2.5e9 elements
    table = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, 1, V - 1, V - 2, 262143, 262144], dtype=torch.int32, device="cuda")
    table[ids.long()] = torch.arange(1, 7, device="cuda").bfloat16()[:, None]
    y = ids[torch.arange(T, device="cuda") % 6].contiguous()
    out = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    print("[offsets] embed", flush=True)
    rbp.policy_embed_fwd(table, y, None, out)
    assert torch.equal(out, table[y.long()])
    del table
    dW = torch.full((V, d), 3.0, device="cuda")
    rbp.policy_embed_bwd(out, y, None, dW, rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V))
    count = torch.bincount(torch.arange(T, device="cuda") % 6).float()
    want = count * torch.arange(1, 7, device="cuda")
    assert torch.equal(dW[ids.long()], want[:, None].expand(6, d))
    dW[ids.long()] = 0.0
    assert not dW.any()
