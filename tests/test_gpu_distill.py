"""policy_distill_fwd_bwd against oracle/vocab.py.

Tolerances, from fp32 arithmetic (e = 2^-24 per rounding): an exponential of y - max is off by
e (2 |y - max| + 4) of itself; a sum of V positive terms, in pieces, by (V / 64 + 64) e at most; so
lse by their sum plus 2 e (|max| + |lse|), each KL term by the errors of its three parts, and a
gradient entry by the relative errors of its exponential and sum plus those of its products.  A
16-bit gradient adds half a step, 2^-8."""

import numpy as np
import pytest
import torch

from gpu_util import require_gpu, to_np
from oracle import vocab
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _cuda(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _case(T, V, K, dtype, seed, use_mass=False, sd=2.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.standard_normal((T, V)) * sd).to(dtype).double().numpy()
    ids = rng.integers(0, V, (T, K)).astype(np.int32)
    lt = (rng.standard_normal((T, K)) * 2 + 6).astype(np.float32)
    mass = (np.log(np.exp(lt.astype(np.float64)).sum(1)) + rng.random(T)).astype(np.float32) \
        if use_mass else None
    B = 1 + T // 7
    seq = np.sort(rng.integers(0, B, T)).astype(np.int32)
    seq[rng.random(T) < 0.15] = -1
    seq_len = rng.integers(1, 50, B).astype(np.int32)
    return z, ids, lt, mass, seq, seq_len, rng


def _run(rbp, z, ids, lt, mass, seq, seq_len, tau=1.0, scale=1.0, dtype=torch.float32, pad=0,
         grad="own", shift=0):
    """grad: "own" tensor, "inplace", or None.  shift: elements the first row is off its
    allocation."""
    T, V = z.shape
    n_seq = len(seq_len) + 3

    def rows(guard, fill):
        flat = guard(shift + T * (V + pad), dtype, float("nan"))
        v = flat[shift:].view(T, V + pad)[:, :V]
        if fill is not None:
            v.copy_(fill)
        return flat, v

    g = Guarded()
    flat_z, zt = rows(g, _cuda(z).to(dtype))
    flat_g, dz = (None, None) if grad is None else (flat_z, zt) if grad == "inplace" else \
        rows(g, None)
    kl, loss, stats = g(T, torch.float32), g(1, torch.float32, 0.5), g(2, torch.float32, 2.0)
    ws = g.ws(rbp.rbp_workspace_bytes(rbp.RBP_OP_DISTILL, T, ids.shape[1], V))
    print(f"[distill] T={T} V={V} K={ids.shape[1]} {dtype} pad={pad} shift={shift} {grad}",
          flush=True)
    rbp.policy_distill_fwd_bwd(zt, _cuda(ids), _cuda(lt), _cuda(mass), _cuda(seq), _cuda(seq_len),
                               n_seq, kl, loss, stats, dz, ws, temperature=tau, scale=scale)
    g.check("distill")
    tau, scale = float(np.float32(tau)), float(np.float32(scale))
    wkl, wloss, wstats, wdz = vocab.distill(z, ids, lt, mass, seq, seq_len, n_seq, tau, scale)
    # per token: error of lse, then of each term
    y = np.where(np.isfinite(z), z, 0.0) / tau
    top = np.abs(y).max(1)
    rel = E * (4 * top + V / 64 + 72)
    tol = np.zeros(T)
    P = np.zeros(T)
    for t in range(T):
        here = ids[t] >= 0
        l = lt[t][here].astype(np.float64) / tau
        if seq[t] < 0 or not np.isfinite(l).any():
            continue
        part = np.abs(np.where(np.isfinite(l), l, 0.0)).max()
        lp = l - (np.log(np.exp(l - l.max()).sum()) + l.max() if mass is None else mass[t])
        p = np.exp(lp)
        P[t] = p.sum()
        live = p > 0
        tol[t] = (p[live] * (rel[t] + E * 8 * (part + top[t] + np.abs(lp[live]) + 16)
                             + E * 8 * (part + 8) * np.abs(lp[live] - y[t, ids[t][here][live]]
                                                           + np.log(V) + top[t]))).sum()
    got = to_np(kl).astype(np.float64)
    assert np.array_equal(np.isfinite(got), np.isfinite(wkl))
    fine = np.isfinite(wkl)
    assert np.all(np.abs(got - wkl)[fine] <= tol[fine])
    w = np.array([scale / (n_seq * seq_len[s]) if s >= 0 else 0.0 for s in seq])
    if fine.all():
        assert abs(loss.item() - 0.5 - wloss) <= (np.abs(w) * (tol + 4 * E * np.abs(wkl))).sum() \
            + 2 * E * (0.5 + abs(wloss))
        assert abs(stats[1].item() - 2 - wstats[1]) <= tol.sum() + 4 * E * (2 + np.abs(wkl).sum())
    assert stats[0].item() == 2 + wstats[0]
    if grad is not None:
        half = 0.0 if dtype == torch.float32 else 2.0 ** -8
        got = to_np(dz.double())
        wide = np.abs(w / tau)[:, None]
        part = np.abs(np.where(np.isfinite(lt), lt, 0)).max(1)[:, None] / tau
        # its two parts are at most |dz| + p_v and p_v
        p = np.zeros_like(z)
        for t in range(T):
            here = (ids[t] >= 0) & (ids[t] < V)
            if seq[t] < 0 or P[t] == 0:
                continue
            l = lt[t][ids[t] >= 0].astype(np.float64) / tau
            norm = np.log(np.exp(l - l.max()).sum()) + l.max() if mass is None else mass[t]
            np.add.at(p[t], ids[t][here], np.exp(lt[t][here].astype(np.float64) / tau - norm))
        p *= wide
        err = (np.abs(wdz) + 2 * p) * (rel[:, None] + E * 8 * (part + 8)) + half * np.abs(wdz) \
            + 2.0 ** -130
        assert np.array_equal(np.isfinite(got), np.isfinite(wdz))
        ok = np.isfinite(wdz)
        assert np.all(np.abs(got - wdz)[ok] <= err[ok] + half * err[ok])
        assert (got[seq < 0] == 0).all()
        # columns behind V and elements before the first row are untouched
        back = flat_g[shift:].view(T, V + pad)[:, V:]
        assert back.isnan().all() and flat_g[:shift].isnan().all()
    return to_np(kl)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 7, 3), (37, 1024, 8), (5, 1000, 256), (9, 63, 64),
                                   (3, 4097, 17), (2, 20000, 5), (33, 513, 65), (4, 33333, 100),
                                   (40, 40001, 9), (64, 8191, 3), (16, 8192, 2)])
def test_divergence_and_gradient(T, V, K, dtype):
    rbp = require_gpu()
    a = _case(T, V, K, dtype, T + V + K)[:6]
    _run(rbp, *a, dtype=dtype)
    _run(rbp, *a, tau=2.5, scale=-0.3, dtype=dtype, grad="inplace")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1, 151936), (3, 152063), (2, 81921), (2, 70000), (2, 163841),
                                 (2, 300007)])
def test_whole_vocabularies(T, V, dtype):
    rbp = require_gpu()
    a = _case(T, V, 20, dtype, V, use_mass=True)[:6]
    a[4][:] = 0
    _run(rbp, *a, dtype=dtype)


def test_many_rows():
    rbp = require_gpu()
    a = _case(1500, 700, 3, torch.bfloat16, 77)[:6]
    _run(rbp, *a, dtype=torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,pad", [(0, 1), (1, 0), (1, 7), (3, 5), (8, 3), (2, 13)])
def test_strides_and_alignments(shift, pad, dtype):
    """Rows of odd lengths, at odd distances, beginning anywhere within 16 bytes."""
    rbp = require_gpu()
    a = _case(6, 2045, 9, dtype, shift + pad, use_mass=True)[:6]
    _run(rbp, *a, dtype=dtype, shift=shift, pad=pad)
    _run(rbp, *a, dtype=dtype, shift=shift, pad=pad, grad="inplace")


def test_a_gradient_aligned_unlike_its_logits():
    rbp = require_gpu()
    for dtype in (torch.float32, torch.bfloat16):
        z, ids, lt, _, seq, seq_len, _ = _case(3, 1003, 4, dtype, 6)
        seq[:] = 0
        both = []
        for off in (0, 1, 3):
            base = torch.zeros(8 + 3 * 1003, dtype=dtype, device="cuda")
            dz = base[off:off + 3 * 1003].view(3, 1003)
            kl, loss, stats = (torch.zeros(n, device="cuda") for n in (3, 1, 2))
            rbp.policy_distill_fwd_bwd(_cuda(z).to(dtype), _cuda(ids), _cuda(lt), None, _cuda(seq),
                                       _cuda(seq_len), 2, kl, loss, stats, dz,
                                       rbp.workspace(rbp.RBP_OP_DISTILL, 3, 4, 1003))
            assert base[:off].eq(0).all() and base[off + 3 * 1003:].eq(0).all()
            both.append(dz.clone())
        assert torch.equal(both[0], both[1]) and torch.equal(both[0], both[2])


def test_absent_entries_and_empty_rows():
    rbp = require_gpu()
    for dtype in (torch.float32, torch.bfloat16):
        z, ids, lt, _, seq, seq_len, rng = _case(12, 500, 6, dtype, 40)
        seq[:] = 0
        ids[0, 3:] = -1
        ids[1, :] = -1                # no teacher
        lt[2, :] = -np.inf            # a teacher without mass
        lt[3, 1:] = -np.inf           # one entry left
        ids[4, :] = 7                 # the same entry six times
        lt[5, 0] = np.nan             # NaN at an absent entry
        ids[5, 0] = -3
        seq[6] = -1                   # masked: whatever it holds
        z[6, :] = np.nan
        lt[6, :] = np.nan
        ids[6, :] = 10 ** 6
        seq[7] = -1
        z[7, :] = np.inf
        z[8, 100:] = -np.inf          # most of the vocabulary masked
        ids[8] = np.arange(6)
        z[9, 100:] = float(torch.finfo(dtype).min)
        ids[9] = np.arange(6)
        z[1, :] = np.nan              # not looked at without a teacher
        _run(rbp, z, ids, lt, None, seq, seq_len, dtype=dtype)
        _run(rbp, z, ids, lt, None, seq, seq_len, dtype=dtype, grad=None)


@pytest.mark.parametrize("V", [300, 20000])
def test_infinite_divergence_and_invalid_values(V):
    """p > 0 where the policy has no mass: KL = inf and a finite gradient; NaN logits, ids behind
    the vocabulary: NaN."""
    rbp = require_gpu()
    z, ids, lt, _, seq, seq_len, _ = _case(5, V, 4, torch.float32, 50)
    seq[:] = 0
    z[0, ids[0, 0]] = -np.inf
    z[1, 17] = np.nan
    ids[2, 1] = V
    ids[3, 2] = 2 ** 31 - 1
    lt[4, 0] = np.nan
    kl, loss, stats = (torch.zeros(n, device="cuda") for n in (5, 1, 2))
    dz = torch.zeros((5, V), device="cuda")
    rbp.policy_distill_fwd_bwd(_cuda(z).float(), _cuda(ids), _cuda(lt), None, _cuda(seq),
                               _cuda(seq_len), 1, kl, loss, stats, dz,
                               rbp.workspace(rbp.RBP_OP_DISTILL, 5, 4, V))
    assert kl[0].item() == np.inf and kl[1:].isnan().all()
    assert dz[0].isfinite().all() and dz[2].isfinite().all() and dz[3].isfinite().all()
    assert dz[1].isnan().all() and dz[4].isnan().all() and loss.isnan().all()


@pytest.mark.parametrize("V", [901, 3001, 8001, 30001, 60001])
def test_large_passes_give_the_rows_of_small_ones(V):
    """Beyond 3/4 GiB the gradient is stored otherwise: the same bits."""
    rbp = require_gpu()
    a = _case(50, V, 5, torch.bfloat16, V)[:6]
    z, ids, lt, _, seq, seq_len = a
    times = (3 << 28) // (50 * V * 2) + 1

    def call(n):
        T = 50 * n
        zt = _cuda(z).bfloat16().repeat(n, 1)
        dz, kl = torch.empty_like(zt), torch.empty(T, device="cuda")
        loss, stats = torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
        rbp.policy_distill_fwd_bwd(zt, _cuda(ids).repeat(n, 1), _cuda(lt).repeat(n, 1), None,
                                   _cuda(seq).repeat(n), _cuda(seq_len), 9, kl, loss, stats, dz,
                                   rbp.workspace(rbp.RBP_OP_DISTILL, T, 5, V))
        return kl.view(n, 50), dz.view(n, 50, V), stats

    print(f"[distill] {times} times 50 rows of {V}", flush=True)
    # rows of an odd length begin at the same place within 16 bytes every 8 rows, and a row's
    # sums run in an order that this place decides: repetitions k and k + 8 are the same
    kl, dz, stats = call(8)  # (400 rows: a block per row)
    big_kl, big_dz, big_stats = call(times)
    assert times >= 16
    for k in range(0, times - 7, 8):
        assert torch.equal(big_kl[k:k + 8], kl) and torch.equal(big_dz[k:k + 8], dz)
    assert big_stats[0].item() == times * stats[0].item() / 8


def test_forward_alone_gives_the_same_divergence():
    rbp = require_gpu()
    a = _case(50, 3001, 12, torch.bfloat16, 60)[:6]
    with_grad = _run(rbp, *a, dtype=torch.bfloat16)
    assert np.array_equal(with_grad, _run(rbp, *a, dtype=torch.bfloat16, grad=None))


def test_gradient_by_differences():
    """Along a direction, in the loss itself (a sum in fp32 of terms known to about 1e-6)."""
    rbp = require_gpu()
    z, ids, lt, _, seq, seq_len, rng = _case(4, 40, 5, torch.float32, 70, sd=1.0)
    seq[:], seq_len[:] = 0, 1
    along = rng.standard_normal(z.shape)

    def call(x, dz):
        kl, loss, stats = (torch.zeros(n, device="cuda") for n in (4, 1, 2))
        rbp.policy_distill_fwd_bwd(_cuda(x).float(), _cuda(ids), _cuda(lt), None, _cuda(seq),
                                   _cuda(seq_len), 1, kl, loss, stats, dz,
                                   rbp.workspace(rbp.RBP_OP_DISTILL, 4, 5, 40), temperature=2.0)
        return loss.item()

    dz = torch.empty((4, 40), device="cuda")
    h = 2.0 ** -6
    call(z, dz)
    slope = (call(z + h * along, None) - call(z - h * along, None)) / (2 * h)
    # the loss is rounded to 2^-24 of about 10, twice; the third derivative of four KLs
    # along a direction of entries up to 3 / tau is below 4 * 27 / 8
    assert abs(slope - (to_np(dz) * along).sum()) < 40 * 2.0 ** -24 / h * 4 + h * h / 6 * 4 * 27 / 8


def test_accumulation_over_calls_is_reproducible():
    rbp = require_gpu()
    z, ids, lt, mass, seq, seq_len, _ = _case(300, 900, 30, torch.bfloat16, 80, use_mass=True)
    args = (_cuda(z).bfloat16(), _cuda(ids), _cuda(lt), _cuda(mass), _cuda(seq), _cuda(seq_len))
    ws = rbp.workspace(rbp.RBP_OP_DISTILL, 300, 30, 900)
    got = []
    for fill in (0, 255):
        ws.fill_(fill)
        kl, loss, stats = (torch.zeros(n, device="cuda") for n in (300, 1, 2))
        dz = torch.empty_like(args[0])
        for _ in range(2):
            rbp.policy_distill_fwd_bwd(*args, 40, kl, loss, stats, dz, ws)
        got.append((kl, loss, stats, dz))
    assert all(torch.equal(a, b) for a, b in zip(*got))
