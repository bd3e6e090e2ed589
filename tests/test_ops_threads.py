"""A plan that several threads call at once, on the CPU: its calls share a workspace, so
each call's launches follow the ones before them whole."""
import threading
import time
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2411_17866_amd import dsm, ops  # noqa: E402


class _Stream:
    cuda_stream = 7

    def wait_stream(self, other):
        pass


@pytest.fixture
def calls(monkeypatch):
    """The binding's calls, replaced by ones that take a while; how many ran at once."""
    state = types.SimpleNamespace(running=0, most=0, count=0)

    def call(*args, **kwargs):
        state.running += 1
        state.count += 1
        state.most = max(state.most, state.running)
        time.sleep(0.002)
        state.running -= 1

    for name in ("dsm_linear_ce", "dsm_orthogonalize", "dsm_ortho_step"):
        monkeypatch.setattr(dsm, name, call)
    monkeypatch.setattr(dsm, "dsm_ce_workspace", lambda problem: 256)
    monkeypatch.setattr(dsm, "dsm_ortho_workspace", lambda problem: 256)
    stream = _Stream()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def allocate(self, workspace_bytes, device):
        self.device, self.workspace_bytes = torch.device("cpu"), workspace_bytes
        self.workspace, self._stream = torch.empty(256, dtype=torch.uint8), stream

    monkeypatch.setattr(ops._Plan, "_allocate", allocate)
    monkeypatch.setattr(ops._Plan, "_on_device", lambda self: __import__("contextlib").nullcontext())
    return state


def _together(work, threads=6, times=5):
    errors = []

    def run():
        try:
            for _ in range(times):
                work()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    pool = [threading.Thread(target=run) for _ in range(threads)]
    for t in pool:
        t.start()
    for t in pool:
        t.join()
    assert not errors, errors[0]


def test_calls_of_one_cross_entropy_follow_each_other(calls):
    plan = ops.LinearCE(3, 4, 5, device="cpu")
    h, w, t = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int64)
    _together(lambda: plan(h, w, t))
    assert calls.count == 30 and calls.most == 1


def test_calls_of_one_orthogonalisation_follow_each_other(calls):
    plan = ops.Ortho(3, 4, 2, device="cpu")
    x, m, g = (torch.zeros(2, 3, 4) for _ in range(3))

    def work():
        plan.orthogonalize(g)
        plan.step(x, m, g, lr=0.1, mu=0.9)
        plan.direction(m, g, g, mu=0.9)

    _together(work)
    assert calls.count == 90 and calls.most == 1


def test_calls_of_two_plans_do_not_wait_for_each_other(calls):
    plans = iter([ops.LinearCE(3, 4, 5, device="cpu") for _ in range(4)])
    h, w, t = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int64)
    lock = threading.Lock()

    def work():
        with lock:
            plan = next(plans)
        plan(h, w, t)

    _together(work, threads=4, times=1)
    assert calls.count == 4
