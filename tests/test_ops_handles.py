"""What an optimiser's handle holds on to, with the native calls stood in for (no GPU needed)."""
import ctypes
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2308_14129_amd import ops


class NoLibrary:
    """The calls of an AdamW handle: every one succeeds and does nothing."""

    def __init__(self):
        self.steps = 0

    def tig_adamw_workspace_bytes(self, cfg, table, n, need):
        need._obj.value = 256
        return 0

    def tig_adamw_create(self, cfg, table, n, ws, bytes, stream, h):
        h._obj.value = 1
        return 0

    def tig_adamw_step(self, *a):
        self.steps += 1
        return 0

    def tig_adamw_destroy(self, h):
        pass


class OnHost:
    def __init__(self, device):
        pass

    def __enter__(self):
        return 0

    def __exit__(self, *a):
        pass


@pytest.fixture
def host(monkeypatch):
    lib = NoLibrary()
    monkeypatch.setattr(ops, "_lib", lambda: lib)
    monkeypatch.setattr(ops, "_On", OnHost)
    return lib


def watched(n, gone, dtype=np.float32):
    """A tensor over an array whose end is noted in `gone`."""
    a = np.zeros(n, dtype=dtype)
    weakref.finalize(a, gone.append, n)
    return torch.from_numpy(a)


@pytest.mark.parametrize("how", ["item", "clear", "data"])
def test_memory_whose_address_the_handle_has_outlives_the_callers_lists(host, how):
    gone = []
    lists = [[watched(10 * k + i, gone) for i in range(1, 4)] for k in range(1, 6)]  # params, grads, m, v, masters: sizes 11 .. 53
    for k in range(1, 5):
        lists[k] = [watched(len(q), gone) for q in lists[0]]
    gc.collect()
    gone.clear()
    opt = ops.AdamW(lists[0], lists[1], lists[2], lists[3], watched(1, gone, np.int64), masters=lists[4])
    for l in lists:
        if how == "item":
            for i in range(len(l)):
                l[i] = torch.ones(len(l[i]))
        elif how == "data":
            for q in l:
                q.data = torch.ones(len(q))
        else:
            l.clear()
    gc.collect()
    assert not gone, "the next step would use freed memory"
    opt.step(1e-3)
    assert host.steps == 1
    opt.close()
    del opt
    gc.collect()
    assert len(gone) == 16


def test_memory_of_8bit_states_is_held_too(host):
    gone = []
    p, g = [watched(300, gone)], [watched(300, gone)]
    m, v = ([watched(300, gone, np.uint8).view(torch.float8_e4m3fn)] for _ in range(2))
    ms, vs = ([watched(2, gone)] for _ in range(2))
    opt = ops.AdamW(p, g, m, v, torch.zeros(1, dtype=torch.int64), m_scales=ms, v_scales=vs)
    for l in (p, g, m, v, ms, vs):
        l.clear()
    gc.collect()
    assert not gone
    del opt
    gc.collect()
    assert len(gone) == 6


class Recorder:
    def __init__(self):
        self.on = []

    def data_ptr(self):
        return 256

    def record_stream(self, stream):
        self.on.append(stream)


def test_a_step_on_another_stream_is_noted_on_the_handles_own_memory(host, monkeypatch):
    """The allocator must not give the list of chunks away while a step on another stream than its own may still read it."""
    now = [7]
    monkeypatch.setattr(OnHost, "__enter__", lambda self: now[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: ("stream", now[0]))
    t = [torch.zeros(10) for _ in range(4)]
    opt = ops.AdamW([t[0]], [t[1]], [t[2]], [t[3]], torch.zeros(1, dtype=torch.int64))
    opt.ws, opt.norm = Recorder(), Recorder()
    opt.step(1e-3)
    assert opt.ws.on == [] and opt.norm.on == []
    now[0] = 8
    opt.step(1e-3)
    now[0] = 7
    opt.step(1e-3)
    assert opt.ws.on == [("stream", 8)] and opt.norm.on == [("stream", 8)]
