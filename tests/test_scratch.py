"""The workspaces that the binding takes for direct calls, without a GPU: stubbed entry points
stand for the library's and record the workspace each call gets."""
import threading
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture
def calls(monkeypatch):
    """Attention calls on tensors in host memory, "device" -1, stream 7."""
    from paper_2607_02501_amd import eb

    monkeypatch.setattr(eb, "_get_device", lambda: -1)
    monkeypatch.setattr(eb, "_raw_stream", lambda dev: 7)
    monkeypatch.setattr(eb, "_capturing", lambda: False)
    monkeypatch.setattr(eb, "_stream", lambda device: 7)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(eb, "_SCRATCH", type(eb._SCRATCH)())
    monkeypatch.setattr(eb, "_attention_ws", lambda op, stream: 1000)
    monkeypatch.setattr(eb, "_ATTN_WS_BYTES", {})
    got = []

    def attention(op, ws, nbytes, stream):
        got.append((ws, nbytes))
        return eb.EB_OK

    monkeypatch.setattr(eb, "_attention", attention)
    cache = SimpleNamespace(k=torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16), index=-1, dim=64, heads=1,
                            dtype=torch.bfloat16, device=torch.device("cpu"), shape=(eb.EB_BF16, 1, 64, 16, 4, 0))
    cache.v = cache.k.clone()
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    table, q_start, kv_len = (torch.tensor(v, dtype=torch.int32) for v in ([[0, 1]], [0, 1], [5]))

    def call():
        return eb.attention(q, cache, table, q_start, kv_len, 1, 32)

    return SimpleNamespace(eb=eb, got=got, call=call)


def test_one_thread_keeps_its_workspace(calls):
    calls.call()
    calls.call()
    assert calls.got[0] == calls.got[1] and calls.got[0][1] >= 1000


def test_threads_have_a_workspace_each(calls, monkeypatch):
    """Calls of two threads on one stream: the launches of either may fall between the other's."""
    barrier, seen = threading.Barrier(2, timeout=20), {}

    def attention(op, ws, nbytes, stream):
        barrier.wait()          # both calls are under way
        seen[threading.get_ident()] = ws
        barrier.wait()
        return calls.eb.EB_OK

    monkeypatch.setattr(calls.eb, "_attention", attention)
    threads = [threading.Thread(target=calls.call) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(30)
    assert len(seen) == 2 and len(set(seen.values())) == 2


def test_capture_on_another_device_than_the_current(calls, monkeypatch):
    """A captured call's workspace belongs to the graph, whichever device is current."""
    eb, current = calls.eb, [0]
    monkeypatch.setattr(eb, "_get_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: current.__setitem__(0, d))
    monkeypatch.setattr(eb, "_capturing", lambda: current[0] == -1)
    calls.call()
    assert not eb._SCRATCH.bufs and current == [0]
    assert calls.got[0][1] == 1000


def test_captured_projections_have_a_workspace_each(calls, monkeypatch):
    """Two graphs captured on one stream may run at the same time."""
    eb, got, kept = calls.eb, [], []
    qw = SimpleNamespace(qtype="q8_0", n=64, k=64, buf=torch.zeros(64, dtype=torch.uint8))
    x, out = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64)
    empty = torch.empty

    def keep(*args, **kw):   # the graph's memory outlives the call
        kept.append(empty(*args, **kw))
        return kept[-1]

    def fused(op, path, ws, nbytes, stream):
        got.append(ws)
        return eb.EB_OK

    monkeypatch.setattr(eb, "_ws_bytes", lambda op, path: 1000)
    monkeypatch.setattr(eb, "_fused_ws", fused)
    monkeypatch.setattr(eb, "_WS_BYTES", {})
    monkeypatch.setattr(torch, "empty", keep)
    for capturing in (False, True, True, False):
        monkeypatch.setattr(eb, "_capturing", lambda: capturing)
        eb._run_op(qw, x, out, eb.EB_BF16, eb.EB_PATH_AUTO)
    assert got[0] == got[3] and len(set(got[:3])) == 3
    monkeypatch.setattr(eb, "_capturing", lambda: True)
    assert eb.scratch("cpu", 1000).data_ptr() != eb.scratch("cpu", 1000).data_ptr()
