"""Which stream an AdamW object waits for (on the host, no GPU needed)."""

import pytest
import torch

gift = pytest.importorskip("paper_2607_07494_amd.gift")


def test_the_null_stream_is_torchs_default_stream(monkeypatch):
    """torch.cuda.ExternalStream(0) is a stream of torch's pool, which nothing of the context's runs on."""
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    for handle, want in ((0, "default"), (0x1230, ("external", 0x1230))):
        c = gift.Context(stream=handle)
        assert gift.AdamW(c, [])._stream() == want
        c.close()
