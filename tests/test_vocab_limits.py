"""The largest and the smallest that the embedding, verification and distillation take, and the
sizes of their workspaces (CPU: the C ABI, stopped by its own checks before any launch)."""

import random

import pytest
import torch

import paper_2604_08706_amd as rbp
from test_vocab_refusals import _distill, _embed_bwd, _verify

LONGEST = 2 ** 31 - 1 - 2 ** 14


@pytest.mark.parametrize("call", [
    lambda V: _verify(V=V, ld=V, ldd=V, ws_bytes=0),
    lambda V: _distill(V=V, ld=V, ws_bytes=0)], ids=["verify", "distill"])
def test_rows_whose_last_tile_passes_31_bits_are_refused(call):
    """Indices beyond the row's end are formed before they are compared with it."""
    assert call(LONGEST) == rbp.RBP_EWORKSPACE  # goes on to the next check
    assert call(LONGEST + 1) == call(2 ** 31 - 1) == rbp.RBP_EUNSUPPORTED


def test_rows_whose_last_chunk_passes_31_bits_are_refused():
    """The gradient counts columns up to the end of a chunk of 512."""
    for T in (1, 60):
        assert _embed_bwd(T=T, d=2 ** 31 - 512, ws_bytes=0) == rbp.RBP_EWORKSPACE
        for d in (2 ** 31 - 504, 2 ** 31 - 8):
            assert _embed_bwd(T=T, d=d, ws_bytes=0) == rbp.RBP_EUNSUPPORTED


def test_gradients_beyond_what_a_launch_counts_are_refused():
    for T, d in ((1 << 30, 136), ((1 << 24) + 1, 1 << 13), (512, (1 << 28) + 8)):
        assert _embed_bwd(T=T, d=d, ws_bytes=0) == rbp.RBP_EUNSUPPORTED
    for T, d in ((1 << 30, 128), (1 << 24, 1 << 13), (512, 1 << 28)):
        assert _embed_bwd(T=T, d=d, ws_bytes=0) == rbp.RBP_EWORKSPACE


def _growing(op, sizes, d, V):
    """rbp_workspace_bytes over growing n."""
    got = [rbp.rbp_workspace_bytes(op, n, d, V) for n in sizes]
    for k in range(1, len(got)):
        assert got[k] >= got[k - 1] > 0, (sizes[k - 1:k + 1], got[k - 1:k + 1], d, V)


def _sizes(top, borders, seed):
    """1 .. 300, both sides of every border, and others between, in order."""
    rng = random.Random(seed)
    sizes = set(range(1, 300)) | {round(top ** rng.random()) for _ in range(3000)}
    for b in borders:
        sizes |= {b - 1, b, b + 1}
    return sorted(n for n in sizes if 1 <= n <= top)


@pytest.mark.parametrize("d", [8, 64, 136, 512, 520, 896, 3584, 8200, 1 << 20])
def test_embedding_gradient_workspace_grows_with_the_batch(d):
    chunks = -(-d // 512) if d > 256 else 1
    borders = [(8 << k) * 4096 // chunks for k in range(7)] + [512, 8192, 12288, 65536]
    _growing(rbp.RBP_OP_EMBED_BWD, _sizes(1 << 27, borders, d), d, 152064)


VOCABULARIES = [1, 1000, 1024, 2047, 2048, 8192, 32768, 65536, 152064, 1 << 28]


@pytest.mark.parametrize("V", VOCABULARIES)
def test_verification_workspace_grows_with_sequences_and_drafts(V):
    for K in (0, 1, 2, 4, 7, 31, 255):
        rows = 2 * K + 1
        borders = [64 // rows, 65 // rows] + [(1 << k) // rows for k in range(15, 25)]
        _growing(rbp.RBP_OP_VERIFY, _sizes(min(1 << 21, (1 << 24) // (K + 1)), borders, V + K), K, V)
    for B in (1, 2, 7, 8, 13, 21, 22, 63, 64, 65, 1000, 30000, 65536):
        got = [rbp.rbp_workspace_bytes(rbp.RBP_OP_VERIFY, B, K, V) for K in range(256)]
        assert all(a <= b for a, b in zip(got, got[1:])), (B, V)


@pytest.mark.parametrize("V", VOCABULARIES)
def test_distillation_workspace_grows_with_tokens_and_entries(V):
    for K in (1, 8, 31, 256):
        _growing(rbp.RBP_OP_DISTILL, _sizes((1 << 22) - 1, [64, V // 512], V + K), K, V)
    for T in (1, 2, 15, 16, 17, 63, 64, 65, 300, 5000):
        got = [rbp.rbp_workspace_bytes(rbp.RBP_OP_DISTILL, T, K, V) for K in range(1, 257)]
        assert all(a <= b for a, b in zip(got, got[1:])), (T, V)


def test_what_sorting_keeps_of_its_blocks_stays_small():
    """Every block reads the digit counts of all: at 2^30 tokens they had been 512 MB for each of
    262144 blocks.  Beside two (key, position) pairs a token and two rows for 256 tokens the
    workspace has room for 2 MB."""
    for T in (1 << 20, (1 << 21) + 1, 1 << 24, 1 << 30):
        got = rbp.rbp_workspace_bytes(rbp.RBP_OP_EMBED_BWD, T, 8, 1000)
        assert got <= 16 * T + (T // 256 + 4097) * 2 * 8 * 4 + (1 << 21)


def test_sizes_that_do_not_fit_the_c_abi_are_refused():
    """2^32 + 10 rows, columns or sequences were taken for 10.  (Tensors without memory.)"""
    many = 2 ** 32 + 10

    def t(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    i, bf = t(4, dtype=torch.int32), torch.bfloat16
    with pytest.raises(ValueError, match="2\\^31"):
        rbp.policy_embed_fwd(t(many, 8, dtype=bf), i, None, t(4, 8, dtype=bf))
    with pytest.raises(ValueError, match="2\\^31"):
        rbp.policy_embed_bwd(t(4, 8), i, None, t(many, 8), None)
    for shape in ((1, 1, many), (many, 1, 4), (1, many, 4)):
        with pytest.raises(ValueError, match="2\\^31"):
            rbp.policy_verify_drafts(t(*shape), None, None, None, i, i, i, i, None)
    with pytest.raises(ValueError, match="2\\^31"):
        rbp.policy_distill_fwd_bwd(t(4, many), i, i, None, i, i, 1, i, i, i, None, None)
