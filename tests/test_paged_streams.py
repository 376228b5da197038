"""Plans of the paged-cache operators on streams other than the one their own tensors were allocated on: the order of
waits and launches with stand-ins for streams (no GPU), and on a GPU with work still pending on the memory."""
import ctypes

import pytest
import torch

import paper_2601_17917_b200 as ds
from paper_2601_17917_b200 import paged

gpu = pytest.mark.gpu
DEV = "cuda:0"


class FakeStream:
    def __init__(self, raw, log, capturing=False):
        self.cuda_stream, self.log, self.capturing, self.device = raw, log, capturing, torch.device("cuda", 0)

    def record_event(self):
        return f"event of {self.cuda_stream}"

    def wait_event(self, event):
        self.log.append((self.cuda_stream, "waits for", event))


class FakeTensor:
    def __init__(self, log):
        self.log = log

    def record_stream(self, stream):
        self.log.append(("kept for", stream.cuda_stream))


@pytest.fixture
def plan_on(monkeypatch):
    def make(log, current, own=1):
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
        monkeypatch.setattr(paged, "_raw_stream", lambda index: current[0].cuda_stream)
        monkeypatch.setattr(paged, "_current_device", lambda: 0)
        monkeypatch.setattr(paged, "_capturing", lambda stream: stream.capturing, raising=False)

        class Lib:
            @staticmethod
            def launch(ref, raw):
                log.append(("launch on", raw))
                return ds.DS_OK
        monkeypatch.setattr(paged, "lib", lambda: Lib)

        class Plan(paged._Plan):
            _name = "launch"
        p = Plan()
        p._ready(ctypes.c_int(0), torch.device("cuda", 0), (), [FakeTensor(log) for _ in range(own)] + [None])
        return p
    return make


def test_a_launch_on_another_stream_waits_for_the_stream_that_the_memory_came_from(plan_on):
    log = []
    here, side = FakeStream(1, log), FakeStream(2, log)
    current = [here]
    p = plan_on(log, current)
    p._enqueue(None)
    p._enqueue(here)
    assert log == [("launch on", 1)] * 2                     # no waiting where the memory is from
    for given in (side, None):                               # named, and as the current one
        log.clear()
        current[0] = side
        p._enqueue(given)
        assert log == [(2, "waits for", "event of 1"), ("launch on", 2), ("kept for", 2)]
    log.clear()
    current[0] = here
    p = plan_on(log, current, own=0)                         # nothing of its own: the caller orders everything
    p._enqueue(side)
    assert log == [("launch on", 2)]


def test_captures_hold_only_waits_of_their_own(plan_on):
    log = []
    here, side = FakeStream(1, log), FakeStream(2, log)
    p = plan_on(log, [here])
    side.capturing = True                                    # made before the capture: no graph can wait for that
    p._enqueue(side)
    assert log == [("launch on", 2), ("kept for", 2)]
    log.clear()
    here.capturing = True                                    # made within it, launched on a fork: a wait in the graph
    p = plan_on(log, [here])
    p._enqueue(side)
    assert log == [(2, "waits for", "event of 1"), ("launch on", 2), ("kept for", 2)]
    log.clear()
    here.capturing = side.capturing = False                  # and after it
    p._enqueue(side)
    assert log == [("launch on", 2), ("kept for", 2)]


@gpu
@pytest.mark.parametrize("form", ["plan", "function"])
def test_memory_with_work_pending_on_it(form):
    """Results and workspace get blocks that were freed on the current stream with kernels still to come that write them;
    the call goes to another stream, whose inputs are ready."""
    g = torch.Generator().manual_seed(0)
    B, Hq, Hkv, D, ps, n = 2, 28, 4, 128, 16, 6000
    per = -(-n // ps)
    q = torch.randn(B, Hq, D, generator=g).bfloat16().to(DEV)
    k, v = (torch.randn(B * per, Hkv, ps, D, generator=g).bfloat16().to(DEV) for _ in range(2))
    table = torch.randperm(B * per, generator=g).view(B, per).to(torch.int32).to(DEV)
    table = torch.cat([table, table, table], 1)              # room: the call is split, with a workspace
    lens = torch.tensor([n, n - 7], dtype=torch.int32, device=DEV)
    args = (q, k, v, table, lens, 0.1)
    need = ds.ds_attn_paged_workspace(*args)
    assert need > 0
    want = ds.ds_attn_paged(*args).clone()
    old, new, lists = (torch.zeros(B, dtype=torch.int32, device=DEV), torch.full((B,), 300, dtype=torch.int32, device=DEV),
                       torch.arange(64, dtype=torch.int32, device=DEV))
    count, block = torch.tensor([64], dtype=torch.int32, device=DEV), torch.zeros(B, 40, dtype=torch.int32, device=DEV)
    want_pages = {n: t.clone() for n, t in ds.ds_page_update(old, new, block.clone(), lists, count, ps, max_rows=5000).items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        stale = [torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty_like(q), torch.empty(5000, dtype=torch.int64, device=DEV),
                 torch.empty(5000, dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)]
        torch.cuda._sleep(100_000_000)                       # some 50 ms
        for t in stale:
            t.fill_(1)
        del stale, t
        if form == "plan":
            got = ds.PagedAttnPlan(*args).launch(side)
        else:
            got = ds.ds_attn_paged(*args, stream=side)
        with torch.cuda.stream(side):
            table_side = torch.zeros(B, 40, dtype=torch.int32, device=DEV)
        make = ds.PageUpdatePlan(old, new, table_side, lists, count, ps, max_rows=5000)
        make.launch(side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        for name, t in want_pages.items():
            assert torch.equal(getattr(make, name), t), name
        del got, make
