"""Calls of several Python threads."""
import threading
import time

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402


def run_beside(work):
    """What `work` returns or raises in a thread of its own."""
    got = []

    def body():
        try:
            got.append(work())
        except Exception as e:  # noqa: BLE001
            got.append(e)
    t = threading.Thread(target=body)
    t.start()
    t.join()
    if isinstance(got[0], Exception):
        raise got[0]
    return got[0]


def test_a_call_of_another_thread_is_made_while_one_is_prepared():
    want, mine, other = pamm.draw_indices_host(1000, 8, 3), torch.zeros(8, dtype=torch.int32), []

    def call():
        other.append(run_beside(lambda: pamm.draw_indices_host(1000, 8, 3)))
        pamm._check(pamm._lib.pamm_draw_indices_host(1000, 8, 3, pamm._ptr(mine)), "draw")

    run = pamm.prepared(call)
    assert torch.equal(other[0], want) and not mine.any()
    run()
    assert torch.equal(mine, want)


def test_two_threads_prepare_at_once():
    outs, both = [torch.zeros(8, dtype=torch.int32) for _ in range(2)], threading.Barrier(2, timeout=30)

    def prepare(i):
        def call():
            both.wait()
            pamm._check(pamm._lib.pamm_draw_indices_host(1000, 8, 10 + i, pamm._ptr(outs[i])), "draw")
            both.wait()
        return pamm.prepared(call)

    runs = [None, None]

    def body(i):
        runs[i] = prepare(i)
    ts = [threading.Thread(target=body, args=(i,)) for i in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert not outs[0].any() and not outs[1].any()
    for i in range(2):
        runs[i]()
        assert torch.equal(outs[i], pamm.draw_indices_host(1000, 8, 10 + i))


@pytest.mark.gpu
def test_an_operator_of_another_thread_runs_while_one_is_prepared():
    x = torch.randn((5, 64), device="cuda")
    table = pamm.rotary_table(5, *pamm.rotary_frequencies(64))
    grads = [torch.randn((70,), device="cuda")]
    # before the threads start: what another thread leaves unmade must not be handed out as the result
    wanted = (pamm.norm_forward(x)[0], pamm.rotary(x.view(5, 1, 64), table), pamm.grad_norm(grads))
    y = torch.zeros_like(x)
    seen = []

    def beside():
        out = torch.zeros((5, 1, 64), device="cuda")
        norm = torch.zeros((), device="cuda")
        return pamm.norm_forward(x, Y=torch.zeros_like(x))[0], pamm.rotary(x.view(5, 1, 64), table, out=out), pamm.grad_norm(grads, norm=norm)

    def call():
        seen.append(run_beside(beside))
        pamm.norm_forward(x, Y=y)

    run = pamm.prepared(call)
    assert all(torch.equal(a, b) for a, b in zip(seen[0], wanted)) and not y.any()
    run()
    assert torch.equal(y, wanted[0])


@pytest.mark.gpu
def test_other_threads_go_on_while_a_call_waits_for_the_launch_queue():
    x = torch.randn((64, 2, 64), device="cuda")
    table = pamm.rotary_table(64, *pamm.rotary_frequencies(64))
    out = torch.empty_like(x)
    pamm.rotary(x, table, out=out)
    torch.cuda.synchronize()
    stop, gap = threading.Event(), [0.0]

    def watch():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            gap[0] = max(gap[0], now - last)
            last = now
    t = threading.Thread(target=watch)
    t.start()
    longest = 0.0
    torch.cuda._sleep(2_000_000_000)            # about a second of the device, which launches queue up behind
    for _ in range(6000):
        start = time.perf_counter()
        pamm.rotary(x, table, out=out)
        longest = max(longest, time.perf_counter() - start)
    stop.set()
    t.join()
    torch.cuda.synchronize()
    assert longest > 0.2, longest               # the queue was full: the call waited
    assert gap[0] < 0.5 * longest, (gap[0], longest)
