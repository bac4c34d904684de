"""Sizes that gift_embedding_grad refuses and what its scratch query says of
them, all on the host (no GPU needed): fake pointers are never dereferenced."""

import ctypes

import pytest
import torch

gift = pytest.importorskip("paper_2607_07494_amd.gift")
FAKE = ctypes.c_void_p(0x1000)


def status(N, T, V, d, accumulate):
    """Of a call with a scratch of 1 byte: past every check of sizes the scratch (or, without a GPU, the device) is refused."""
    ctx = gift.Context(stream=0)
    st = gift.LIB.gift_embedding_grad(ctx.handle, FAKE, 0, FAKE, 0, N, T, V, d, 1.0, accumulate, FAKE, FAKE, 1)
    text = gift.LIB.gift_last_error().decode()
    ctx.close()
    return st, text


@pytest.mark.parametrize("N,T,V,d,writes,adds", [
    (2, 100, 8, 8, True, True),
    (65535, 1, 1 << 30, 8, False, True),              # the rows to clear
    (65535, 32768, 8, 1 << 20, False, False),         # the runs' columns
    (1, (1 << 31) - 1, 8, 300, False, False),
    (1, (1 << 31) - 1, 8, 256, False, False),         # one chunk of columns, ...
    (1, (1 << 31) - 4096, 8, 256, True, True),        # ... and the most positions it takes, nearly
    (1, 1 << 20, (1 << 31) - 2, 1 << 20, False, False),
    (1, 64, (1 << 31) - 2, 64, False, True),
])
def test_scratch_is_0_where_both_forms_are_refused(N, T, V, d, writes, adds):
    for accumulate, taken in ((0, writes), (1, adds)):
        st, text = status(N, T, V, d, accumulate)
        assert (st != gift.ESHAPE) == taken, text
        assert st != gift.OK and (taken or "more work" in text)
    assert (gift.embedding_grad_scratch(N, T, V, d) > 0) == (writes or adds)


def test_a_number_of_ranks_past_32_bits_is_not_taken_modulo(monkeypatch):
    seen = []

    class Library:
        def gift_embedding_grad(self, *args):
            seen.append(args[5])
            return gift.OK

    N = (1 << 32) + 1
    assert gift.embedding_grad_scratch(N, 4, 4, 4) == 0
    monkeypatch.setattr(gift, "LIB", Library())
    monkeypatch.setattr(gift, "_on_current_device", lambda **tensors: None)

    class Context:
        _h = None

    def meta(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    gift.embedding_grad(Context(), meta(N, 1, dtype=torch.int32), meta(N, 1, 2), meta(N, 3, 2))
    assert ctypes.c_int32(seen[0]).value > 65535       # refused by the library
