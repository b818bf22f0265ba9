"""policy_embed_fwd and policy_embed_bwd against oracle/vocab.py, at the sizes and tokens where
they can go wrong.

Tolerances: a bf16 value is off by half a step, 2^-8 of it (and the fp32 product before it by
2^-24); a sum of n fp32 terms, in any order, by n 2^-24 of the sum of their magnitudes, plus the
scale's product, the addition to what was there and the rounding of each."""

import numpy as np
import pytest
import torch

from gpu_util import require_gpu, to_np
from oracle import vocab
from test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24
BF16 = 2.0 ** -8


def _tokens(kind, T, V, rng):
    if kind == "one":
        y = np.full(T, V - 1)
    elif kind == "distinct":
        y = rng.permutation(max(T, V))[:T] % V
    elif kind == "runs":  # runs that end and begin everywhere within slices and tiles
        y = np.sort(rng.integers(0, max(2, T // 40), T)) % V
        y = y[rng.permutation(T)]
    else:  # skewed: half the batch is one token
        y = np.where(rng.random(T) < 0.5, V // 2, rng.integers(0, V, T))
    return y.astype(np.int32)


def _seq(T, rng, share=0.2):
    return np.where(rng.random(T) < share, -1, rng.integers(0, 5, T)).astype(np.int32)


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("T,d,V,scale,masked", [
    (1, 8, 1, 1.0, False), (1, 64, 1024, 8.0, False), (7, 896, 500, 0.5, True),
    (513, 72, 4097, 1.7, True), (300, 3584, 77, 1.0, False), (4099, 8, 11, 59.866, True),
    (1203, 3584, 300, 0.7, True)])
def test_lookup(T, d, V, scale, masked):
    rbp = require_gpu()
    rng = np.random.default_rng(T + d)
    table = torch.from_numpy(rng.standard_normal((V, d)) * 0.02).to(torch.bfloat16)
    y = _tokens("skewed", T, V, rng)
    seq = _seq(T, rng) if masked else None
    g = Guarded()
    out = g((T, d), torch.bfloat16)
    rbp.policy_embed_fwd(table.cuda(), _cuda(y), None if seq is None else _cuda(seq), out,
                         scale=scale)
    g.check("embed_fwd")
    want = vocab.embed(table.double().numpy(), y, seq, float(np.float32(scale)))
    got = to_np(out.double())
    assert np.all(np.abs(got - want) <= np.abs(want) * BF16 * (1 + 2.0 ** -15))


def test_ids_outside_the_table():
    """A row of NaN where not masked; a masked one is not looked at."""
    rbp = require_gpu()
    table = torch.ones((10, 16), dtype=torch.bfloat16, device="cuda")
    y = torch.tensor([3, 10, -1, 2 ** 31 - 1, -2 ** 31, -5], dtype=torch.int32, device="cuda")
    seq = torch.tensor([0, 0, 0, 0, 0, -1], dtype=torch.int32, device="cuda")
    out = torch.zeros((6, 16), dtype=torch.bfloat16, device="cuda")
    rbp.policy_embed_fwd(table, y, seq, out)
    assert out[0].eq(1).all() and out[1:5].isnan().all() and out[5].eq(0).all()
    dW = torch.zeros((10, 16), device="cuda")
    dx = torch.full((6, 16), float("nan"), device="cuda")
    dx[0] = 2.0
    rbp.policy_embed_bwd(dx, y, seq, dW, rbp.workspace(rbp.RBP_OP_EMBED_BWD, 6, 16, 10))
    assert dW[3].eq(2).all() and dW.abs().sum().item() == 32


def _check_backward(rbp, T, d, V, kind, dtype, acc, scale=1.0, masked=True):
    rng = np.random.default_rng([T, d, V])
    y, seq = _tokens(kind, T, V, rng), _seq(T, rng) if masked else None
    dx = torch.from_numpy(rng.standard_normal((T, d))).to(dtype)
    start = rng.standard_normal((V, d)).astype(np.float32)
    g = Guarded()
    dW = g((V, d), torch.float32, torch.from_numpy(start))
    ws = g.ws(rbp.rbp_workspace_bytes(rbp.RBP_OP_EMBED_BWD, T, d, V))
    args = (dx.cuda(), _cuda(y), None if seq is None else _cuda(seq))
    print(f"[embed] T={T} d={d} V={V} {kind} {dtype} accumulate={acc}", flush=True)
    rbp.policy_embed_bwd(*args, dW, ws, scale=scale, accumulate_dW=acc)
    g.check("embed_bwd")
    s = float(np.float32(scale))
    x = dx.double().numpy()
    want = vocab.embed_backward(x, y, seq, V, s, start if acc else None)
    size = vocab.embed_backward(np.abs(x), y, seq, V, abs(s), np.abs(start) if acc else None)
    live = np.ones(T, bool) if seq is None else seq >= 0
    count = np.bincount(y[live], minlength=V)[:, None]
    assert np.all(np.abs(to_np(dW) - want) <= (count + 2) * F32 * size)
    if acc:  # rows without a token are left as they were
        none = np.nonzero(count[:, 0] == 0)[0]
        assert np.array_equal(to_np(dW)[none], start[none])
    again = torch.from_numpy(start).cuda()
    rbp.policy_embed_bwd(*args, again, ws, scale=scale, accumulate_dW=acc)
    assert torch.equal(again, dW)
    return dW


@pytest.mark.parametrize("kind", ["one", "distinct", "runs", "skewed"])
@pytest.mark.parametrize("T,d,V", [(1, 8, 1), (31, 64, 1000), (33, 24, 5), (257, 136, 4097),
                                   (4095, 8, 600), (4097, 16, 151936), (8193, 40, 262144),
                                   (20001, 8, 300001)])
def test_gradient(T, d, V, kind):
    _check_backward(require_gpu(), T, d, V, kind, torch.float32, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("T,d,V", [(100, 896, 511), (777, 3584, 512), (65, 1536, 513),
                                   (2050, 512, 2049), (1025, 520, 64)])
def test_gradient_types_widths_and_modes(T, d, V, dtype, acc):
    _check_backward(require_gpu(), T, d, V, "runs", dtype, acc, scale=-3.3)


@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("kind", ["one", "distinct", "runs", "skewed"])
@pytest.mark.parametrize("T,d,V,dtype", [
    (512, 520, 1025, torch.float32), (512, 8, 70001, torch.bfloat16), (511, 128, 3, torch.float32),
    (5, 8200, 70, torch.bfloat16), (2, 256, 5000, torch.float32), (513, 128, 1000, torch.float32)])
def test_gradient_of_few_tokens(T, d, V, dtype, kind, acc):
    """Up to 512 tokens, summed without a sort, and the first count beyond them."""
    _check_backward(require_gpu(), T, d, V, kind, dtype, acc, scale=0.7)


def test_gradient_of_a_long_batch():
    """Many tiles of the sort and slices of the sums; half the batch is one token."""
    _check_backward(require_gpu(), 150001, 8, 5000, "skewed", torch.bfloat16, False, masked=False)


def test_no_token_and_only_masked_tokens():
    rbp = require_gpu()
    for acc in (False, True):
        dW = torch.full((7, 8), 3.0, device="cuda")
        none = torch.zeros(0, dtype=torch.int32, device="cuda")
        rbp.policy_embed_bwd(torch.zeros((0, 8), device="cuda"), none, none, dW, None,
                             accumulate_dW=acc)
        assert dW.eq(3.0 if acc else 0.0).all()
        dW.fill_(3.0)
        y = torch.zeros(40, dtype=torch.int32, device="cuda")
        rbp.policy_embed_bwd(torch.full((40, 8), float("inf"), device="cuda"), y, y - 1, dW,
                             rbp.workspace(rbp.RBP_OP_EMBED_BWD, 40, 8, 7), accumulate_dW=acc)
        assert dW.eq(3.0 if acc else 0.0).all()


def test_gradient_by_differences():
    """d/dtable of sum(r * lookup) along a direction, on values that are exact in bf16."""
    rbp = require_gpu()
    rng = np.random.default_rng(5)
    V, d, T, scale = 60, 16, 500, 0.5
    table = torch.from_numpy(rng.integers(-64, 64, (V, d))).to(torch.bfloat16).cuda()
    step = torch.from_numpy(rng.integers(0, 2, (V, d))).to(torch.bfloat16).cuda()
    y = torch.from_numpy(rng.integers(0, V, T).astype(np.int32)).cuda()
    r = torch.from_numpy(rng.integers(-8, 8, (T, d))).float().cuda()
    out = [torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rbp.policy_embed_fwd(table + step, y, None, out[0], scale=scale)
    rbp.policy_embed_fwd(table - step, y, None, out[1], scale=scale)
    dW = torch.empty((V, d), device="cuda")
    rbp.policy_embed_bwd(r, y, None, dW, rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V), scale=scale)
    difference = ((out[0].double() - out[1].double()) * r.double()).sum().item() / 2
    assert difference == (dW.double() * step.double()).sum().item()  # small integers: exact


@pytest.mark.parametrize("T,d,V,kind,acc", [
    (4096, 24, 700, "runs", True), (8192, 16, 5000, "skewed", True), (8192, 8, 3, "distinct", True),
    (8191, 8, 9000, "one", False), (12288, 448, 150001, "one", False),
    (12287, 448, 150001, "skewed", False)])
def test_gradient_sorted_by_counting(T, d, V, kind, acc):
    """The most tokens of each rule, whole blocks and the last one short."""
    _check_backward(require_gpu(), T, d, V, kind, torch.bfloat16, acc)


@pytest.mark.parametrize("T,d,V,kind", [(7001, 448, 150001, "skewed"), (12289, 448, 150001, "runs"),
                                        (6145, 8, 511, "runs"), (20001, 24, 512, "skewed"),
                                        (600001, 8, 900, "runs")])
def test_gradient_written_whole_on_every_route(T, d, V, kind):
    """Counting beside the clearing of dW; tiles with one, two and three digits; the longest
    slices."""
    _check_backward(require_gpu(), T, d, V, kind, torch.float32, False)


def test_gradient_of_a_table_with_four_digits():
    rbp = require_gpu()
    V, d, T = (1 << 27) + 3, 8, 9001
    rng = np.random.default_rng(8)
    ids = np.unique(np.concatenate([rng.integers(0, V, 300), [0, V - 1, 1 << 26, (1 << 27) - 1]]))
    y = ids[rng.integers(0, len(ids), T)].astype(np.int32)
    dx = rng.standard_normal((T, d)).astype(np.float32)
    dW = torch.zeros((V, d), device="cuda")
    rbp.policy_embed_bwd(_cuda(dx), _cuda(y), None, dW,
                         rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V), accumulate_dW=True)
    place = np.searchsorted(ids, y)
    want = vocab.embed_backward(dx, place, None, len(ids))
    size = vocab.embed_backward(np.abs(dx), place, None, len(ids))
    count = np.bincount(place, minlength=len(ids))[:, None]
    rows = torch.from_numpy(ids).cuda()
    assert np.all(np.abs(to_np(dW[rows]) - want) <= (count + 2) * F32 * size)
    dW[rows] = 0.0
    assert not dW.any()
