"""The embedding, verified drafts and distillation where a program reuses what it has: one
workspace for batches of every size, and other calls that the tests of each operator do not make."""

import numpy as np
import pytest
import torch
from scipy.sparse import csr_matrix

from gpu_util import require_gpu, to_np
from oracle import vocab

pytestmark = pytest.mark.gpu


def _rows_summed(y, dx, V):
    """fp64 [V, d] on the host: the sums of dx over equal y.  (Atomic 64-bit additions to one
    row, as an indexed addition on the GPU makes them, take 20 s for 160000 of them.)"""
    one = csr_matrix((np.ones(len(y)), (to_np(y), np.arange(len(y)))), shape=(V, len(y)))
    return torch.from_numpy(one @ to_np(dx).astype(np.float64))


def test_embedding_gradients_of_many_sizes_in_the_workspace_of_the_largest():
    rbp = require_gpu()
    rng = np.random.default_rng(1)
    V, d, most = 700, 512, 40000
    ws = rbp.workspace(rbp.RBP_OP_EMBED_BWD, most, d, V)
    dx = torch.from_numpy(rng.integers(-4, 5, (most, d)).astype(np.float32)).cuda()
    y = torch.from_numpy(np.where(rng.random(most) < 0.5, 3, rng.integers(0, V, most))
                         .astype(np.int32)).cuda()
    # (4096 slices of 8 positions at 32768 tokens, more than the largest batch has)
    for T in (1, 513, 4097, 8193, 12289, 32768, 32769, most):
        ws.fill_(255)
        dW = torch.full((V, d), 7.0, device="cuda")
        print(f"[workspace] embed_bwd T={T}", flush=True)
        rbp.policy_embed_bwd(dx[:T], y[:T], None, dW, ws)
        # small integers: exact
        assert torch.equal(dW.double().cpu(), _rows_summed(y[:T], dx[:T], V))


def test_verification_of_a_shrinking_batch_in_one_workspace():
    """Sequences and drafts fall away: more segments a row from 64 rows on."""
    rbp = require_gpu()
    B, K, V = 40, 4, 33000
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    z = torch.randn((B, K + 1, V), generator=g, device="cuda") * 2
    zd = z[:, :K] + 0.5 * torch.randn((B, K, V), generator=g, device="cuda")
    pick = torch.rand((B, K, V), generator=g, device="cuda").log_().neg_().log_().neg_()
    x = (zd + pick).argmax(-1).int()
    u = torch.rand((B, K + 1), generator=g, device="cuda")
    ws = rbp.workspace(rbp.RBP_OP_VERIFY, B, K, V)
    for b, k in ((40, 4), (21, 1), (8, 4), (7, 4), (1, 4), (32, 0), (3, 2)):
        ws.fill_(255)
        tokens = torch.empty((b, k + 1), dtype=torch.int32, device="cuda")
        logp = torch.empty((b, k + 1), device="cuda")
        n = torch.empty(b, dtype=torch.int32, device="cuda")
        print(f"[workspace] verify B={b} K={k}", flush=True)
        for draft in (zd, None):
            zk = z[:b, :k + 1].contiguous()
            dk = None if draft is None or k == 0 else draft[:b, :k].contiguous()
            uk = u[:b, :k + 1].contiguous()
            rbp.policy_verify_drafts(zk, dk, x[:b, :k].contiguous(), None, uk, tokens, logp, n, ws)
            for i in (0, b - 1):
                want, lp = vocab.verify(to_np(zk[i].double()),
                                        None if dk is None else to_np(dk[i].double()),
                                        to_np(x[i, :k]), k, to_np(uk[i]).astype(np.float64))
                assert tokens[i, :len(want)].tolist() == want and n[i].item() == len(want)
                assert np.abs(to_np(logp[i, :len(want)]) - lp).max() < 1e-5


def test_distillation_of_a_shrinking_batch_in_one_workspace():
    """Rows shared by blocks from 64 on down, in the workspace of a batch that has none."""
    rbp = require_gpu()
    rng = np.random.default_rng(5)
    T, V, K = 200, 33000, 100
    ws = rbp.workspace(rbp.RBP_OP_DISTILL, T, K, V)
    z = torch.from_numpy(rng.standard_normal((T, V)).astype(np.float32)).cuda()
    ids = torch.from_numpy(rng.integers(0, V, (T, K)).astype(np.int32)).cuda()
    lt = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda()
    seq = torch.zeros(T, dtype=torch.int32, device="cuda")
    length = torch.ones(1, dtype=torch.int32, device="cuda")
    for t in (200, 65, 64, 33, 16, 15, 1):
        ws.fill_(255)
        kl, loss, stats = (torch.zeros(n, device="cuda") for n in (t, 1, 2))
        dz = torch.empty((t, V), device="cuda")
        print(f"[workspace] distill T={t}", flush=True)
        rbp.policy_distill_fwd_bwd(z[:t], ids[:t], lt[:t], None, seq[:t], length, 1, kl, loss, stats,
                                   dz, ws)
        rows = [0, t - 1]
        wkl, _, _, wdz = vocab.distill(to_np(z[rows].double()), to_np(ids[rows]), to_np(lt[rows]),
                                       None, [0, 0], [1], 1)
        # KL terms of about 16 in fp32; gradients of exponentials off by 2^-24 (2 |y| + 4)
        assert np.abs(to_np(kl[rows]) - wkl).max() < 2e-5 and stats[0].item() == t
        assert np.abs(to_np(dz[rows]) - wdz).max() < 1e-6


@pytest.mark.parametrize("shift", [100.0, -1000.0, 30000.0])
@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("T,V", [(70, 3000), (3, 20000)])
@pytest.mark.parametrize("use_mass", [False, True])
def test_divergence_does_not_depend_on_a_constant_in_the_logits(T, V, tau, shift, use_mass):
    """All values are multiples of 2^-7 below 2^15, so that the shifted ones are exact.  An
    exponential of y - max is off by 2^-24 (2 |y - max| + 4), a sum of positive terms in pieces by
    (V / 64 + 64) of them, the teacher's part likewise, wherever the logits lie; a teacher's sum
    that is given is taken as it is.  Blocks of their own and rows shared by blocks."""
    rbp = require_gpu()
    rng = np.random.default_rng(int(V + abs(shift)))
    K = 9
    z = np.round(rng.standard_normal((T, V)) * 2 * 128) / 128
    lt = np.round((rng.standard_normal((T, K)) * 2 + 6) * 128) / 128
    ids = rng.integers(0, V, (T, K)).astype(np.int32)
    tau = float(np.float32(tau))
    # (multiples of 128 over tau would not be exact: the sum is shifted in 64 bits, rounded once)
    mass = np.log(np.exp(lt / tau).sum(1)) + 0.5 + shift / tau if use_mass else None
    mass = None if mass is None else mass.astype(np.float32)
    z, lt = z + shift, lt + shift
    assert np.array_equal(z.astype(np.float32), z) and np.array_equal(lt.astype(np.float32), lt)
    kl, loss, stats = (torch.zeros(n, device="cuda") for n in (T, 1, 2))
    rbp.policy_distill_fwd_bwd(
        torch.from_numpy(z).float().cuda(), torch.from_numpy(ids).cuda(),
        torch.from_numpy(lt).float().cuda(), None if mass is None else torch.from_numpy(mass).cuda(),
        torch.zeros(T, dtype=torch.int32, device="cuda"),
        torch.ones(1, dtype=torch.int32, device="cuda"), 1, kl, loss, stats, None,
        rbp.workspace(rbp.RBP_OP_DISTILL, T, K, V), temperature=tau)
    wkl, wloss, _, _ = vocab.distill(z, ids, lt, mass, [0] * T, [1], 1, tau)
    spread = (z.max() - z.min() + lt.max() - lt.min()) / tau
    P = 1.0 if mass is None else \
        np.exp((lt - lt.max()) / tau + (lt.max() / tau - mass[:, None].astype(np.float64))).sum(1)
    # its exponentials, its sum, and the roundings of what is left, below 2 spread + 16
    tol = P * 2.0 ** -24 * (2 * spread + 4 + V / 64 + 64 + 4 * (2 * spread + 16))
    assert np.all(np.abs(to_np(kl) - wkl) <= tol)
    assert abs(loss.item() - wloss) <= np.sum(tol) + 2.0 ** -22 * abs(wloss)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,pad", [(1, 0), (3, 0), (0, 3), (2, 5)])
def test_shared_rows_with_a_gradient_aligned_unlike_its_logits(dtype, off, pad):
    """Few long rows, whose blocks then store element by element: the bits of an aligned gradient,
    and nothing beside it."""
    rbp = require_gpu()
    rng = np.random.default_rng(off + pad)
    T, V, K = 5, 9001, 7
    z = torch.from_numpy(rng.standard_normal((T, V))).to(dtype).cuda()
    ids = torch.from_numpy(rng.integers(0, V, (T, K)).astype(np.int32)).cuda()
    ids[:, 0], ids[:, 1] = 0, V - 1  # loose elements of the row's ends
    lt = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda()
    seq = torch.tensor([0, 0, -1, 0, 0], dtype=torch.int32, device="cuda")
    length = torch.ones(1, dtype=torch.int32, device="cuda")
    ws = rbp.workspace(rbp.RBP_OP_DISTILL, T, K, V)

    def call(logits, dz):
        kl, loss, stats = (torch.zeros(n, device="cuda") for n in (T, 1, 2))
        rbp.policy_distill_fwd_bwd(logits, ids, lt, None, seq, length, 1, kl, loss, stats, dz, ws)
        return kl

    # rows at one place of 16 bytes each in the logits; the gradient `off` elements on
    wide = torch.full((T, V + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:, :V] = z
    want = torch.empty((T, V + pad), dtype=dtype, device="cuda")
    kl = call(wide[:, :V], want[:, :V])
    flat = torch.full((off + T * (V + pad) + 8,), 7.0, dtype=dtype, device="cuda")
    dz = flat[off:off + T * (V + pad)].view(T, V + pad)
    print(f"[shared] {dtype} off={off} pad={pad}", flush=True)
    assert torch.equal(call(wide[:, :V], dz[:, :V]), kl)
    assert torch.equal(dz[:, :V], want[:, :V])
    assert dz[:, V:].eq(7).all() and flat[:off].eq(7).all() and flat[off + T * (V + pad):].eq(7).all()
    _, _, _, exact = vocab.distill(to_np(z.double()), to_np(ids), to_np(lt), None, to_np(seq), [1], 1)
    half = 0.0 if dtype == torch.float32 else 2.0 ** -8
    # exponentials off by 2^-24 (2 |y| + 4) of themselves and sums by 2^-24 (V / 64 + 64), beside
    # the teacher's probabilities of at most 1
    assert np.all(np.abs(to_np(dz[:, :V].double()) - exact)
                  <= half * np.abs(exact) + 2.0 ** -24 * 300 * (np.abs(exact) + (exact < 0)))


def _verify_one_draft(rbp, z, zd, x, u):
    """Tokens emitted first, and their number, of one fp32 draft per row of z [B, 2, V]."""
    B, _, V = z.shape
    tokens = torch.empty((B, 2), dtype=torch.int32, device="cuda")
    logp, n = torch.empty((B, 2), device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    rbp.policy_verify_drafts(torch.from_numpy(z).float().cuda(), torch.from_numpy(zd).float().cuda(),
                             torch.from_numpy(x).cuda(), None, torch.from_numpy(u).cuda(), tokens,
                             logp, n, rbp.workspace(rbp.RBP_OP_VERIFY, B, 1, V))
    return to_np(tokens)[:, 0], to_np(n)


def test_draws_from_a_small_remainder_beside_the_borders_of_segments():
    """Totals of max(p - q, 0) around 1e-7: the drawn token's step of the exact running sum holds u
    but for 2^-25 + 1e-12 / total, which the header states.  (64 segments of a row: the borders
    between them and their neighbours, where a segment's error would show.)"""
    rbp = require_gpu()
    rng = np.random.default_rng(11)
    B, V = 20, 70001
    z = rng.standard_normal((B, 2, V)).astype(np.float32).astype(np.float64)
    zd, x = z[:, :1].copy(), np.zeros((B, 1), np.int32)
    u = np.full((B, 2), 0.99, np.float32)
    run = []
    for i in range(B):
        x[i, 0] = rng.integers(0, V)
        z[i, 0, x[i, 0]] = zd[i, 0, x[i, 0]] = -2.0
        zd[i, 0, x[i, 0]] += 0.05 * (1 + i % 4)
        e = [np.exp(a.astype(np.longdouble)) for a in (z[i, 0], zd[i, 0])]
        rest = np.maximum(e[0] / e[0].sum() - e[1] / e[1].sum(), 0)
        run.append((np.cumsum(rest / rest.sum()), float(rest.sum())))
        at = (V * int(rng.integers(1, 64))) // 64 + i % 3 - 1
        u[i, 1] = np.float32(run[i][0][at])
    tokens, n = _verify_one_draft(rbp, z, zd, x, u)
    assert (n == 1).all()
    for i, (cdf, total) in enumerate(run):
        assert 1e-8 < total < 1e-6 and tokens[i] != x[i, 0]
        off = 2.0 ** -25 + 1e-12 / total
        low = cdf[tokens[i] - 1] if tokens[i] > 0 else 0
        assert low - off <= u[i, 1] <= cdf[tokens[i]] + off, (i, total)


def test_a_remainder_below_the_sums_own_error_counts_as_none():
    """One fp32 step more at the draft's logit leaves about 1e-12, a few times what the two sums are
    off by: the token is drawn from p, so with u inside the draft's own step it is the draft's."""
    rbp = require_gpu()
    rng = np.random.default_rng(12)
    B, V = 8, 20001
    z = rng.standard_normal((B, 2, V)).astype(np.float32)
    zd, x = z[:, :1].copy(), rng.integers(0, V, (B, 1)).astype(np.int32)
    u = np.full((B, 2), 1 - 2.0 ** -24, np.float32)
    for i in range(B):
        z[i, 0, x[i, 0]] = zd[i, 0, x[i, 0]] = -1.5
        zd[i, 0, x[i, 0]] = np.nextafter(np.float32(-1.5), np.float32(0))
        p = vocab.distribution(z[i, 0].astype(np.float64))
        q = vocab.distribution(zd[i, 0].astype(np.float64))
        assert float(u[i, 0]) * q[x[i, 0]] > p[x[i, 0]] * (1 + 2.0 ** -25)  # rejected
        assert q[x[i, 0]] - p[x[i, 0]] < 2.0 ** -36
        u[i, 1] = np.float32(p[:x[i, 0]].sum() + 0.5 * p[x[i, 0]])
    tokens, n = _verify_one_draft(rbp, z.astype(np.float64), zd.astype(np.float64), x, u)
    assert (n == 1).all() and (tokens == x[:, 0]).all()


@pytest.mark.parametrize("T,V,kind,acc", [
    ((1 << 21) - 1, 300001, "skewed", True), ((1 << 21) + 1, 5000, "uniform", False),
    ((1 << 21) + 4097, 300001, "skewed", False), (3145733, 5000, "equal", True),
    ((1 << 22) + 5, 511, "uniform", True)])
def test_embedding_gradient_of_more_tokens_than_the_sort_has_tiles_at_once(T, V, kind, acc):
    """From 2^21 tokens on a sorting block takes two tiles and more, the last of them cut short or
    empty.  Small integers: every sum is exact."""
    rbp = require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    if kind != "uniform":
        y[torch.rand(T, generator=g, device="cuda") < (2.0 if kind == "equal" else 0.5)] = V // 3
    seq = torch.randint(-1, 4, (T,), generator=g, device="cuda", dtype=torch.int32)
    dx = torch.randint(-4, 5, (T, 8), generator=g, device="cuda").float()
    dW = torch.randint(-9, 10, (V, 8), generator=g, device="cuda").float()
    keep = seq >= 0
    want = _rows_summed(y[keep], dx[keep], V) + (dW.double().cpu() if acc else 0.0)
    ws = rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, 8, V)
    ws.fill_(255)
    print(f"[sort] T={T} V={V} {kind} {acc}", flush=True)
    rbp.policy_embed_bwd(dx, y, seq, dW, ws, accumulate_dW=acc)
    assert torch.equal(dW.double().cpu(), want)


def test_embedding_gradient_of_few_rows_that_are_very_long():
    """512 rows of 2^24 columns and some, 17 GB: a block for each chunk of each row would be more
    threads than a launch has.  Small integers: exact."""
    rbp = require_gpu()
    T, V, d = 512, 2, (1 << 24) + 8
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    line = torch.randint(-3, 4, (d,), generator=g, device="cuda").bfloat16()
    times = torch.randint(-2, 3, (T,), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dx = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    for t in range(T):
        torch.mul(line, times[t], out=dx[t])
    dW = torch.full((V, d), 7.0, device="cuda")
    print("[few] 512 long rows", flush=True)
    rbp.policy_embed_bwd(dx, y, None, dW, rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V),
                         accumulate_dW=True)
    for v in range(V):
        assert torch.equal(dW[v], 7.0 + line.float() * times[y == v].float().sum())


def _accepted(rbp, z, x, tau):
    """Log-probs of drafts from the policy's own rows z [B, K + 1, V], all of them accepted."""
    B, K1, V = z.shape
    tokens = torch.empty((B, K1), dtype=torch.int32, device="cuda")
    logp, n = torch.empty((B, K1), device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    rbp.policy_verify_drafts(z, z[:, :K1 - 1].contiguous(), torch.from_numpy(x).cuda(), None,
                             torch.full((B, K1), 0.5, device="cuda"), tokens, logp, n,
                             rbp.workspace(rbp.RBP_OP_VERIFY, B, K1 - 1, V), temperature=tau)
    assert (n == K1).all() and np.array_equal(to_np(tokens)[:, :K1 - 1], x)
    return to_np(logp)[:, :K1 - 1].astype(np.float64)


# Of the sum: exponentials off by 1.43 2^-24, three additions of eight, 2^-24 each, and what is
# left of the rounding of log2 e / temperature, 2^-24 of it, on elements that lie (weighted) log2 8
# powers of two below the largest of their eight at most: 3 ln 2 2^-24.  Then the output's rounding,
# half a step of its value.
def _close(got, want):
    return np.all(np.abs(got - want) <= (1.43 + 3 + 3 * np.log(2)) * 2.0 ** -24 + 2.0 ** -24 * np.abs(want) + 1e-9)


def test_log_probs_of_accepted_drafts_over_a_flat_vocabulary():
    """Equal logits that hold 0.8 between them, the first 256 of every 2048 nearly 8 powers of two
    below: a rounding of the others' distance from those would be the same for all, 6e-7 at this
    temperature.  The draft is a token that holds the rest."""
    rbp = require_gpu()
    B, V, tau = 12, 1 << 17, 2.5
    low, flat = float(np.float32(-3.1)), float(np.float32(10.718529))
    z = np.full((B, 2, V), flat)
    z.reshape(B, 2, -1, 2048)[..., :256] = low
    top = float(np.float32(flat + tau * np.log(V * 7 / 8 / 4)))
    x = (256 + 2048 * np.arange(B) + 5 * np.arange(B)).astype(np.int32)[:, None]
    for i in range(B):
        z[i, :, x[i, 0]] = top
    rest = (V * 7 / 8 - 1) * np.exp((flat - top) / tau) + V / 8 * np.exp((low - top) / tau)
    got = _accepted(rbp, torch.from_numpy(z).float().cuda(), x, tau)
    print("[log-probs] largest error", np.abs(got + np.log1p(rest)).max())
    assert _close(got, -np.log1p(rest))


def test_log_probs_of_accepted_drafts_where_a_row_begins_far_below_zero():
    """The first 256 of every 2048 logits are nearly 64 powers of two below the others, which lie
    beside 0: their difference from those would be rounded to 2^-18, by the same for all."""
    rbp = require_gpu()
    B, V = 12, 1 << 17
    low = np.float32(-46.0)
    near = (np.float32(-1.71) + np.arange(4000, dtype=np.float32) * np.float32(2.0 ** -23))
    lost = np.abs((near - low).astype(np.float64) - (near.astype(np.float64) - float(low)))
    flat = float(near[lost.argmax()])
    assert lost.max() > 1.8e-6
    z = np.full((B, 2, V), flat)
    z.reshape(B, 2, -1, 2048)[..., :256] = low
    x = (256 + 2053 * np.arange(B)).astype(np.int32)[:, None]
    top = float(np.float32(flat + np.log(V * 7 / 8 / 4)))
    for i in range(B):
        z[i, :, x[i, 0]] = top
    rest = (V * 7 / 8 - 1) * np.exp(flat - top) + V / 8 * np.exp(float(low) - top)
    got = _accepted(rbp, torch.from_numpy(z).float().cuda(), x, 1.0)
    print("[log-probs] largest error", np.abs(got + np.log1p(rest)).max())
    assert _close(got, -np.log1p(rest))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0.0, 50.0, -55.0, 1e3, -1e5])
@pytest.mark.parametrize("tau,sd", [(1.0, 3.0), (1.3, 20.0), (0.2, 0.5)])
def test_log_probs_of_accepted_drafts_wherever_the_logits_lie(dtype, offset, tau, sd):
    """Rows around 0, whose reference is 0, beside the borders where it is not, and far away; ends
    of a row masked by -infinity and by the type's lowest value."""
    rbp = require_gpu()
    rng = np.random.default_rng(int(abs(offset) + 10 * sd))
    B, K, V = 3, 2, 20011
    tau = float(np.float32(tau))
    z = torch.from_numpy(rng.standard_normal((B, K + 1, V)) * sd + offset).to(dtype)
    z[1, :, :9000] = -np.inf
    z[2, :, 11000:] = torch.finfo(dtype).min
    z[0, 0, :64] = -2e4 if offset > -1e5 else -3e5  # a first piece far below the others
    zd = z.double().numpy()
    x = np.zeros((B, K), np.int32)
    want = np.zeros((B, K))
    for i in range(B):
        for k in range(K):
            p = vocab.distribution(zd[i, k], tau)
            x[i, k] = vocab.draw(p, rng.random())
            want[i, k] = np.log(p[x[i, k]])
    assert _close(_accepted(rbp, z.cuda(), x, tau), want)


@pytest.mark.parametrize("V", [300, 20000])
def test_divergence_from_rows_without_a_distribution(V):
    """Logits of -infinity only, with +infinity or a NaN: the divergence and the row's gradient are
    NaN, and the rows beside them as they would be."""
    rbp = require_gpu()
    rng = np.random.default_rng(V)
    z = rng.standard_normal((5, V)).astype(np.float32)
    ids = rng.integers(0, V, (5, 6)).astype(np.int32)
    lt = rng.standard_normal((5, 6)).astype(np.float32)
    z[1], z[2, V // 2], z[3, 5] = -np.inf, np.inf, np.nan
    kl, loss, stats = (torch.zeros(n, device="cuda") for n in (5, 1, 2))
    dz = torch.zeros((5, V), device="cuda")
    rbp.policy_distill_fwd_bwd(torch.from_numpy(z).cuda(), torch.from_numpy(ids).cuda(),
                               torch.from_numpy(lt).cuda(), None,
                               torch.zeros(5, dtype=torch.int32, device="cuda"),
                               torch.ones(1, dtype=torch.int32, device="cuda"), 1, kl, loss, stats,
                               dz, rbp.workspace(rbp.RBP_OP_DISTILL, 5, 6, V))
    assert kl[1:4].isnan().all() and dz[1:4].isnan().all() and stats[0].item() == 5
    wkl, _, _, wdz = vocab.distill(z[[0, 4]], ids[[0, 4]], lt[[0, 4]], None, [0, 0], [1], 1)
    assert np.abs(to_np(kl[[0, 4]]) - wkl).max() < 2e-5
    assert np.abs(to_np(dz[[0, 4]]) - wdz).max() < 1e-6
