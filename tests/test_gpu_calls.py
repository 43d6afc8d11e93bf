"""What the short calls owe the program around them: other threads, and automatic differentiation."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def test_other_threads_run_while_a_launch_waits(B):
    """A second and a half of work in front, and more launches than a queue holds: a call waits, the interpreter does not."""
    x = torch.randn(32, 256, device="cuda")
    codes, scales = B.checkpoint_store(x)
    torch.cuda._sleep(1000)
    torch.cuda.synchronize()
    t = time.perf_counter()
    torch.cuda._sleep(100_000_000)
    torch.cuda.synchronize()
    a_second = int(100_000_000 / (time.perf_counter() - t))
    gaps, stop = [0.0], threading.Event()

    def watch():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            gaps[0] = max(gaps[0], now - last)
            last = now

    watcher = threading.Thread(target=watch)
    watcher.start()
    time.sleep(0.05)
    torch.cuda._sleep(3 * a_second // 2)
    t = time.perf_counter()
    for _ in range(4000):
        B.checkpoint_store(x, codes=codes, scales=scales)
    waited = time.perf_counter() - t
    stop.set()
    watcher.join()
    torch.cuda.synchronize()
    assert waited > 0.5  # (the queue was full; clocks may have risen since the work was measured)
    assert gaps[0] < 0.5 * waited, (gaps[0], waited)


def test_tensors_that_ask_for_gradients(B):
    """Refused where gradients are recorded, wherever they stand; taken under no_grad and inside an autograd.Function, which brings the backward call."""
    q = torch.randn(40, 2, 64, device="cuda")
    k, v = torch.randn_like(q), torch.randn_like(q).requires_grad_()
    for call in (lambda: B.attention_forward(q, k, v), lambda: B.rotary(v), lambda: B.rotary(q, v), lambda: B.attention_forward(q, k, k, o=v)):
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == 6
        with torch.no_grad():
            call()

    class Attend(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse = B.attention_forward(q, k, v)
            ctx.save_for_backward(q, k, v, o, lse)
            return o

        @staticmethod
        def backward(ctx, d_o):
            q, k, v, o, lse = ctx.saved_tensors
            return B.attention_backward(d_o.contiguous(), q, k, v, o, lse)

    v = torch.randn(40, 2, 64, device="cuda").requires_grad_()
    w = torch.randn_like(q)
    o = Attend.apply(q, k, v)
    o.backward(w)
    with torch.no_grad():
        o, lse = B.attention_forward(q, k, v)
        assert torch.equal(v.grad, B.attention_backward(w, q, k, v, o, lse)[2])


def test_calls_of_several_threads(B):
    """Four threads, each on its own stream, all operators at once: what one thread alone gets."""
    x = torch.randn(200, 256, device="cuda").bfloat16()
    q = torch.randn(300, 4, 64, device="cuda")

    def calls():
        act, codes, scales = B.checkpoint_gelu(x)
        out = [act, codes, scales, B.checkpoint_gelu_backward(x, codes, scales)]
        for t in (q, q.bfloat16()):
            a, b = B.rotary(t, t.clone(), period=100)
            o, lse = B.attention_forward(a, b, t, sequences=3)
            out += [a, b, o, lse, *B.attention_backward(t, a, b, t, o, lse, sequences=3)]
        return out

    alone = calls()
    torch.cuda.synchronize()
    results, errors = [None] * 4, []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    results[i] = calls()
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(alone, r))
