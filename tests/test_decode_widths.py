"""A vocabulary wider than the logits that hold it is refused before the library is called (CPU only: the library is a stand-in)."""
import types

import pytest


def test_sample_of_more_columns_than_there_are(monkeypatch):
    import torch

    import paper_2609_14636_gb300 as stride
    from paper_2609_14636_gb300 import decode

    widths = []
    monkeypatch.setattr(decode, "_dtype", lambda t, name: 1)
    monkeypatch.setattr(stride, "_NATIVE", types.SimpleNamespace(sample=lambda *a: None))
    monkeypatch.setattr(stride, "_dev", lambda t, *a, **k: None)
    monkeypatch.setattr(stride, "_stream", lambda s: None)
    monkeypatch.setattr(stride, "lib", lambda: types.SimpleNamespace(stride_sample=lambda x, dt, ld, V, *a: widths.append((ld, V)) or 0))
    for rows in (1, 3):
        x, tokens = torch.zeros(rows, 128)[:, 28:], torch.zeros(rows, dtype=torch.int32)
        for V in (None, 100, 64):
            decode.stride_sample(x, None, tokens, temperature=0, V=V)
        for V in (101, 128):
            with pytest.raises(ValueError, match="V"):
                decode.stride_sample(x, None, tokens, temperature=0, V=V)
    assert widths == [(128, 100), (128, 100), (128, 64)] * 2
