"""policy_verify_drafts against oracle/vocab.py: tokens and counts equal, log-probs to their
rounding (fp32: half a step, 2^-24 of the value; the 64-bit sums before it are off by less than
1e-9).  Beside draft logits the log-probs of accepted drafts come from 32-bit exponentials: one
of argument y (in powers of two) is off by 3 2^-24 ln 2 |y| for the roundings of the difference,
the factor and the product, and by 2^-23 for its own; weighted by the probabilities |y| is at most
log2 V, plus the 8 that the reference may lag and the 8 by which it then moves, 18 + 16 here, so
the log of the sum is off by 34 * 3 * 2^-24 * 0.7 + 4 * 2^-23 < 5e-6 (the last term: exponentials of
moves, and three additions of eight)."""

import numpy as np
import pytest
import torch

from gpu_util import require_gpu, to_np
from oracle import vocab
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu


def _cuda(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _compare(tokens, logp, n, z, zd, x, n_draft, u, tau):
    B, K1 = tokens.shape
    for i in range(B):
        drafts = K1 - 1 if n_draft is None else min(int(n_draft[i]), K1 - 1)
        if drafts < 0:
            assert n[i] == 0 and (tokens[i] == -1).all() and (logp[i] == 0).all()
            continue
        want, lp = vocab.verify(z[i], None if zd is None else zd[i], None if x is None else x[i],
                                drafts, u[i].astype(np.float64), tau)
        m = len(want)
        assert n[i] == m and tokens[i, :m].tolist() == want, (i, want, tokens[i])
        assert (tokens[i, m:] == -1).all() and (logp[i, m:] == 0).all()
        lp = np.array(lp)
        assert np.array_equal(np.isnan(logp[i, :m]), np.isnan(lp))
        ok = ~np.isnan(lp)
        sums = np.full(m, 1e-9 if zd is None else 5e-6)
        sums[m - 1] = 1e-9
        assert np.all(np.abs(logp[i, :m] - lp)[ok] <= (2.0 ** -24 * np.abs(lp) + sums)[ok])


def _run(rbp, z, zd, x, n_draft, u, tau=1.0, dtype=torch.float32, pad=0):
    """z [B, K + 1, V] float64 holding values of dtype; pad: elements between rows."""
    B, K1, V = z.shape

    def rows(a):
        if a is None:
            return None
        wide = torch.full(a.shape[:2] + (V + pad,), float("nan"), dtype=dtype, device="cuda")
        wide[..., :V] = _cuda(a).to(dtype)
        return wide[..., :V]

    g = Guarded()
    tokens, n = g((B, K1), torch.int32, 77), g(B, torch.int32, 77)
    logp = g((B, K1), torch.float32, 77.0)
    ws = g.ws(rbp.rbp_workspace_bytes(rbp.RBP_OP_VERIFY, B, K1 - 1, V))
    print(f"[verify] B={B} K={K1 - 1} V={V} {dtype} drafts={zd is not None} pad={pad}", flush=True)
    args = (rows(z), rows(zd), _cuda(x), _cuda(n_draft), _cuda(u))
    rbp.policy_verify_drafts(*args, tokens, logp, n, ws, temperature=tau)
    g.check("verify")
    got = to_np(tokens), to_np(logp), to_np(n)
    _compare(*got, z, zd, x, n_draft, u, tau)
    return got


def _values(shape, sd, dtype, rng):
    return torch.from_numpy(rng.standard_normal(shape) * sd).to(dtype).double().numpy()


def _case(B, K, V, dtype, drafted, seed, sd=2.0):
    rng = np.random.default_rng(seed)
    z = _values((B, K + 1, V), sd, dtype, rng)
    zd = torch.from_numpy(z[:, :K] + 0.5 * rng.standard_normal((B, K, V))).to(dtype).double() \
        .numpy() if K else None
    x = np.zeros((B, K), np.int32)
    for i in range(B):
        for k in range(K):
            x[i, k] = vocab.draw(vocab.distribution(zd[i, k] if drafted else z[i, k]), rng.random())
    u = rng.random((B, K + 1)).astype(np.float32)
    return z, zd if drafted else None, x if K else None, u, rng


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 2, 2), (5, 1, 63), (4, 3, 65), (2, 7, 1000),
                                   (9, 4, 1025), (3, 2, 8191), (2, 1, 20001), (2, 2, 151937),
                                   (30, 1, 70001), (24, 1, 200003), (2, 255, 50)])
def test_verified_tokens(B, K, V, drafted, dtype):
    rbp = require_gpu()
    z, zd, x, u, rng = _case(B, K, V, dtype, drafted, B + K + V)
    _run(rbp, z, zd, x, None, u, dtype=dtype)
    n_draft = rng.integers(-1, K + 3, B).astype(np.int32)
    _run(rbp, z, zd, x, n_draft, u, 0.75, dtype, pad=3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V", [(1, 1), (1, 7), (200, 300), (3, 4096), (5, 70001), (1, 400001),
                                 (70, 70001)])
def test_sampling_without_drafts(B, V, dtype):
    rbp = require_gpu()
    z, _, _, u, _ = _case(B, 0, V, dtype, True, V)
    _run(rbp, z, None, None, None, u, 1.5, dtype, pad=5)


def test_many_draws_beside_steps_of_a_flat_distribution():
    """Equal weights: with V a power of two the running sums and u V are exact, so u at a
    step belongs to the next token, and the fp32 below it to the one before."""
    rbp = require_gpu()
    V = 1 << 14
    at = np.array([1, 2, 63, 64, 65, 4095, 4096, 8191, 8192, 12345, V - 1])
    step = (at / V).astype(np.float32)
    u = np.concatenate([step, np.nextafter(step, np.float32(0)), np.zeros(1, np.float32)])
    tokens, _, _ = _run(rbp, np.zeros((len(u), 1, V)), None, None, None, u[:, None])
    assert tokens[:, 0].tolist() == at.tolist() + (at - 1).tolist() + [0]


def test_acceptance_at_the_border():
    """u at p / q itself, and one fp32 step to either side, on many pairs."""
    rbp = require_gpu()
    B, V = 600, 40
    z, zd, x, u, rng = _case(B, 1, V, torch.float32, True, 3)
    for i in range(B):
        p, q = vocab.distribution(z[i, 0]), vocab.distribution(zd[i, 0])
        r = np.float32(min(1.0, p[x[i, 0]] / q[x[i, 0]]))
        u[i, 0] = (np.nextafter(r, np.float32(0)), r, np.nextafter(r, np.float32(2)))[i % 3]
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    _run(rbp, z, zd, x, None, u)


def test_acceptance_at_the_border_over_a_vocabulary():
    """As above over 20001 tokens and through several drafts: the rough sums do not decide."""
    rbp = require_gpu()
    B, K, V = 8, 3, 20001
    z, zd, x, u, _ = _case(B, K, V, torch.bfloat16, True, 4)
    for i in range(B):
        for k in range(K):
            p, q = vocab.distribution(z[i, k]), vocab.distribution(zd[i, k])
            r = np.float32(min(1.0, p[x[i, k]] / q[x[i, k]]))
            u[i, k] = np.nextafter(r, np.float32(0)) if k < i % 3 else np.nextafter(r, np.float32(2))
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    _run(rbp, z, zd, x, None, u, dtype=torch.bfloat16)


def test_weights_left_by_a_draft_that_is_nearly_the_policy():
    """p / q is 1 + 1e-6 and less on all tokens but the draft's: the rough sums do not know
    which is larger, and the draw has to."""
    rbp = require_gpu()
    B, V = 12, 20001
    rng = np.random.default_rng(21)
    z = _values((B, 2, V), 1.0, torch.float32, rng)
    x = np.argmin(z[:, :1], axis=2).astype(np.int32)
    zd = z[:, :1].copy()
    for i in range(B):  # masses of 1e-6 and more
        zd[i, 0, x[i, 0]] += 1.0 + i / 4
        if i % 3 == 0:
            zd[i, 0, rng.integers(0, V, 300)] += 1.0
    zd = torch.from_numpy(zd).float().double().numpy()
    u = rng.random((B, 2)).astype(np.float32)
    u[:, 0] = 0.99
    _, _, n = _run(rbp, z, zd, x, None, u)
    assert (n == 1).all()


def test_nothing_left_of_an_identical_draft():
    """A draft that is no token is rejected, and where the two rows are one (at other
    alignments, so that their sums differ by roundings) the token is drawn from p."""
    rbp = require_gpu()
    z, _, _, u, _ = _case(9, 1, 5003, torch.float32, False, 22)
    x = np.full((9, 1), -1, np.int32)
    _, _, n = _run(rbp, z, z[:, :1].copy(), x, None, u)
    assert (n == 1).all()


def test_identical_draft_and_policy_accept_everything():
    rbp = require_gpu()
    z, _, x, u, _ = _case(6, 5, 777, torch.bfloat16, False, 8)
    u[:, :5] = 1 - 2.0 ** -24
    _, _, n = _run(rbp, z, z[:, :5].copy(), x, None, u, dtype=torch.bfloat16)
    assert (n == 6).all()


def test_masked_vocabulary_and_rows_without_a_distribution():
    rbp = require_gpu()
    inf, nan = np.inf, np.nan
    low = float(torch.finfo(torch.float32).min)
    z, zd, x, u, _ = _case(12, 2, 300, torch.float32, True, 12)
    z[0, :, 10:] = -inf                   # few tokens left
    z[1, :, :] = -inf
    z[1, :, 299] = -3.0                   # one token left
    z[2, :, ::2] = low                    # masked by the type's lowest value
    z[3, 0, :] = -inf                     # no token at the first position
    z[4, 1, 7] = nan                      # no distribution at the second
    z[5, 0, 7] = inf
    z[6, 2, :] = -inf                     # none behind the last draft
    zd[7, 0, :] = -inf                    # none of the draft's
    zd[8, 0, 3] = nan
    zd[9, :, 20:] = -inf                  # a draft that knows 20 tokens
    x[9] = 3
    x[10, 0], x[11, 1] = -1, 300          # no tokens
    u[6, :2] = 0.0
    u[4, 0] = 0.0
    _run(rbp, z, zd, x, None, u)
    _run(rbp, z, None, x, None, u, 0.5)
    z[:] = np.where(z == low, float(torch.finfo(torch.bfloat16).min), z)
    z = torch.from_numpy(z).bfloat16().double().numpy()
    zd = torch.from_numpy(zd).bfloat16().double().numpy()
    _run(rbp, z, zd, x, None, u, dtype=torch.bfloat16, pad=1)


def test_peaked_logits_and_large_values():
    rbp = require_gpu()
    z, zd, x, u, _ = _case(8, 2, 5000, torch.float32, True, 21, sd=30.0)
    _run(rbp, z, zd, x, None, u)
    z[:] = np.float32(1e4) + z
    z = z.astype(np.float32).astype(np.float64)
    _run(rbp, z, zd, x, None, u)
    big = np.array([3e38, -3e38, 3e38, 0.0])[None, None].repeat(2, 0)
    _run(rbp, big.astype(np.float32).astype(np.float64), None, None, None,
         np.array([[0.4], [0.6]], np.float32))


def test_the_end_of_the_unit_interval():
    """The largest u below 1, and values outside [0, 1), draw the last token of positive weight
    or the first."""
    rbp = require_gpu()
    z = np.zeros((5, 1, 3001))
    z[:, :, 2900:] = -np.inf
    z[:, :, :3] = -np.inf
    u = np.array([1 - 2.0 ** -24, 1.0, 7.0, -1.0, 0.0], np.float32)[:, None]
    tokens, _, _ = _run(rbp, z, None, None, None, u)
    assert tokens[:, 0].tolist()[1:] == [2899, 2899, 3, 3]


def test_repeated_calls_and_workspace_contents():
    rbp = require_gpu()
    z, zd, x, u, _ = _case(16, 3, 3333, torch.bfloat16, True, 30)
    a = [_cuda(v) for v in (z, zd, x, u)]
    a[0], a[1] = a[0].bfloat16(), a[1].bfloat16()
    ws = rbp.workspace(rbp.RBP_OP_VERIFY, 16, 3, 3333)
    got = []
    for fill in (0, 255, 171):
        ws.fill_(fill)
        out = [torch.empty((16, 4), dtype=torch.int32, device="cuda"),
               torch.empty((16, 4), device="cuda"),
               torch.empty(16, dtype=torch.int32, device="cuda")]
        rbp.policy_verify_drafts(a[0], a[1], a[2], None, a[3], *out, ws)
        got.append(out)
    for out in got[1:]:
        assert all(torch.equal(p, q) for p, q in zip(got[0], out))


@pytest.mark.parametrize("drafted", [True, False])
def test_logits_far_from_zero(drafted):
    """Around 1e8 an fp32 step is 8, and the exponent of the largest logit would not fit the table's
    arithmetic."""
    rbp = require_gpu()
    rng = np.random.default_rng(41)
    B, K, V = 12, 2, 3000
    z = 1e8 + 8.0 * rng.integers(-3, 1, (B, K + 1, V))
    z[B // 2:] *= -1.0
    zd = z[:, :K] + 8.0 * rng.integers(-1, 2, (B, K, V))
    x = rng.integers(0, V, (B, K)).astype(np.int32)
    u = (rng.random((B, K + 1)) * 1.2 - 0.2).clip(0).astype(np.float32)
    _run(rbp, z, zd if drafted else None, x, None, u)
    _run(rbp, z, zd if drafted else None, x, None, u, 16.0, pad=1)


@pytest.mark.parametrize("offset", [1e5, -3e6, 1e9])
def test_draft_logits_far_from_the_policy_s(offset):
    """The same distributions but for the offset's rounding (0.008, 0.25, 64): which of p and q
    is larger does not show in 32-bit differences of logits."""
    rbp = require_gpu()
    B, K, V = 10, 2, 20001
    z, zd, x, u, _ = _case(B, K, V, torch.float32, True, 61)
    zd = (zd + offset).astype(np.float32).astype(np.float64)
    u[::2, 0] = 1 - 2.0 ** -24
    _run(rbp, z, zd, x, None, u)
    _run(rbp, zd[:, [0, 1, 1]], z[:, :2], x, None, u, pad=1)


@pytest.mark.parametrize("tau", [2.0 ** -100, 1e-3, 300.0, 1e30])
def test_extreme_temperatures(tau):
    rbp = require_gpu()
    tau = float(np.float32(tau))
    for drafted in (True, False):
        z, zd, x, u, _ = _case(7, 2, 1000, torch.float32, drafted, 51)
        z[0, :, 7:] = -np.inf
        _run(rbp, z, zd, x, None, u, tau)
