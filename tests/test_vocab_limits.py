"""The largest and the smallest that the embedding, verification and distillation take, and the
sizes of their workspaces (CPU: the C ABI, stopped by its own checks before any launch)."""

import pytest

import paper_2604_08706_amd as rbp
from test_vocab_refusals import _distill, _verify

LONGEST = 2 ** 31 - 1 - 2 ** 14


@pytest.mark.parametrize("call", [
    lambda V: _verify(V=V, ld=V, ldd=V, ws_bytes=0),
    lambda V: _distill(V=V, ld=V, ws_bytes=0)], ids=["verify", "distill"])
def test_rows_whose_last_tile_passes_31_bits_are_refused(call):
    """Indices beyond the row's end are formed before they are compared with it."""
    assert call(LONGEST) == rbp.RBP_EWORKSPACE  # goes on to the next check
    assert call(LONGEST + 1) == call(2 ** 31 - 1) == rbp.RBP_EUNSUPPORTED
