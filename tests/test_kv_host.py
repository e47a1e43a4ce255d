"""Host-side rules of the key/value cache calls that need no GPU."""
import types

import pytest
import torch

from paper_2309_14717_b200 import binding as Q
from paper_2309_14717_b200 import build as _build


@pytest.fixture(scope="module", autouse=True)
def _built():
    _build.build()


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("batch,max_new,group", [(24, 1, 1), (24, 4, 4), (1, 16, 1), (3, 2, 8), (40, 1, 16)])
def test_scratch_of_few_rows_does_not_vanish_when_m_is_a_bound(batch, max_new, group, scores):
    """m bounds the rows: where no sequence has many, the kernel of few rows runs whatever m says."""
    d = Q.kv_desc(32, 32 // group, 128, 64, 4096)
    exact = Q.qalora_kv_attention_workspace_bytes(d, batch, batch * max_new, max_new, 2048, scores)
    for m in (batch * max_new + 1, batch * max_new + max_new, 2 * batch * max_new + 16, 4096):
        assert Q.qalora_kv_attention_workspace_bytes(d, batch, m, max_new, 2048, scores) >= exact


def test_stream_without_the_raw_handle(monkeypatch):
    """A torch that does not offer the raw handle of its current stream: the stream object's is taken."""
    t = torch.zeros(1)
    monkeypatch.setattr(Q, "_current_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=77, device=device))
    assert Q._kv_stream(None, t) == 77
    assert Q._kv_stream(types.SimpleNamespace(cuda_stream=5), t) == 5
    monkeypatch.setattr(Q, "_current_stream", lambda device: 9)
    assert Q._kv_stream(None, t) == 9


def test_scratch_is_allocated_not_cleared(monkeypatch):
    """Its content may be undefined: only the status word is set."""
    def dirty(*shape, **kw):
        return torch.full(shape if isinstance(shape[0], int) else shape[0], 0xAB, **kw)

    monkeypatch.setattr(torch, "empty", dirty)
    d = Q.kv_desc(8, 2, 128, 64, 100)
    ws = Q.alloc_kv_workspace(d, 3, 6, 2, 1000, True, device="cpu")
    assert ws.numel() == Q.qalora_kv_attention_workspace_bytes(d, 3, 6, 2, 1000, True)
    assert Q.workspace_status(ws) == 0 and (ws[256:] == 0xAB).all()
