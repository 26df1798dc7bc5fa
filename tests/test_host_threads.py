"""Two host threads that enqueue calls of one object: each call gets its own tensors' addresses.  The library's entries are stood in for, so no device is needed."""
import threading

import pytest
import torch

from paper_2507_06517_b200 import binding as B
from paper_2507_06517_b200.pipeline import SpindleKVPagedCache, SpindleKVPromptAttention


def both(monkeypatch, entry, addresses_of, call, sets):
    """Thread 0 is held up just ahead of the library's entry while thread 1 makes its whole call; what the entry got, by thread."""
    got, inside, done = {}, threading.Event(), threading.Event()
    name = threading.local()

    def raw_stream(_):
        if getattr(name, "is", None) == 0:
            inside.set()
            done.wait(0.5)                       # (a call that keeps the other one out goes on after this)
        return 0

    monkeypatch.setattr(B, "current_device", lambda: None)
    monkeypatch.setattr(B, "raw_stream", raw_stream)
    monkeypatch.setattr(B, entry, lambda *a, **kw: got.__setitem__(getattr(name, "is", None), addresses_of(a)))

    def thread(i):
        setattr(name, "is", i)
        if i:
            inside.wait(5)
        call(*sets[i])
        if i:
            done.set()

    call(*sets[0])                               # the layouts are known by now
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(10)
    return got


def test_rotated_appends_of_two_threads(monkeypatch):
    cache = SpindleKVPagedCache(1, 2, None, 2, 64, 4, 2, device="cpu")
    rope = torch.zeros((8, 32, 2))
    sets = [[torch.zeros((1, 2, h, 3, 64)) for h in (2, 2, 2, 4, 4)] for _ in range(2)]
    got = both(monkeypatch, "spindlekv_paged_append_rotated", lambda a: [a[i].ptr for i in (4, 5, 9, 11, 12)],
               lambda K, V, K_out, Q, Q_out: cache.append_rotated(K, V, rope, K_out=K_out, Q=Q, Q_out=Q_out), sets)
    for i in range(2):
        assert got[i] == [t.data_ptr() for t in sets[i]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_attention_of_two_threads(monkeypatch, dtype):
    a = SpindleKVPromptAttention(B.Batch(1, 2, 5, 10), 4, 2, 64, dtype, device="cpu")
    sets = [[torch.zeros((1, 2, h, 5, 64), dtype=dtype) for h in (4, 2, 2, 4)] for _ in range(2)]
    got = both(monkeypatch, "spindlekv_prompt_attend", lambda x: [t.ptr for t in x[6:10]], lambda q, K, V, out: a.run(q, K, V, out=out), sets)
    for i in range(2):
        assert got[i] == [t.data_ptr() for t in sets[i]]
