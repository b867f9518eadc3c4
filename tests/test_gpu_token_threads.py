"""Calls from several host threads at once: they have nothing in common."""

import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_two_vocabularies_in_two_threads():
    """Rows of both sizes are kept in shared memory by the same kernel, in different amounts."""
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_1802_04819_b200 as slaq
    slaq.build()
    work, failed = [], []
    for vocab in (128_000, 50_001):
        x = torch.randn(200, vocab, device="cuda").bfloat16()
        t = torch.randint(vocab, (200,), device="cuda")
        g = torch.full((200,), -1 / 200, device="cuda")
        work.append((x, t, g, slaq.token_loss(x, t, g), torch.cuda.Stream()))
    torch.cuda.synchronize()

    def calls(x, t, g, want, stream):
        try:
            with torch.cuda.stream(stream):
                out = torch.empty_like(x)
                for _ in range(3000):
                    logprob, _ = slaq.token_loss(x, t, g, out=out)
                stream.synchronize()
            if not (torch.equal(logprob, want[0]) and torch.equal(out, want[1])):
                failed.append("other results")
        except Exception as e:   # noqa: BLE001 - the test says what it was
            failed.append(repr(e))
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=calls, args=w) for w in work]
        for th in threads:
            th.start()
        for th in threads:
            th.join()
    finally:
        sys.setswitchinterval(interval)
    assert not failed, failed
