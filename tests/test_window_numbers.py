"""Numbers of a window that do not fit the C interface's 32 bits are refused by the binding instead of being cut off (no GPU here)."""
import types

import pytest

from paper_2506_19651_b200 import binding as pb
from paper_2506_19651_b200 import build as pbuild


@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32, 2 ** 32 + 100, -2 ** 32 + 100, 2 ** 63 - 1])
def test_window(window, monkeypatch):
    import torch
    pbuild.build()
    monkeypatch.setattr(pb, "_stream", lambda: None)
    s, g = pb.make_shape(4, 1, 0, 1, 4, 2, 64), pb.make_pages(8, 16, 4, 2)
    x, ws = torch.empty(0), types.SimpleNamespace(nbytes=1 << 20, data_ptr=lambda: 4096)
    for call in (lambda: pb.pevlm_window_attn(s, window, x, x, x, 50, 0, 54, x, x, ws),
                 lambda: pb.pevlm_packed_attn(s, g, window, ws, ws, ws, ws, ws, 0, 0, ws, ws, ws)):
        with pytest.raises(pb.PevlmError) as e:  # (of no rows: nothing is launched where the number is taken)
            call()
        assert e.value.code == pb.PEVLM_EINVAL
