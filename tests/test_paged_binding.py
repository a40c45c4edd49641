"""The Python binding of the paged calls and the clipping: what it keeps between
calls, shared by threads and devices.  No GPU: device queries are replaced."""
import sys
import threading

import pytest
import torch

import paper_2608_11368_amd as pair


@pytest.fixture
def one_stream(monkeypatch):
    monkeypatch.setattr(pair, "_status_words", {})
    monkeypatch.setattr(pair, "_stream", lambda stream: 7)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)


def test_the_last_status_word_taken_by_another_thread(one_stream):
    """Between the look at the words and the taking of one, another thread of the
    same stream takes the last."""
    class Taken(list):
        def pop(self):
            self.clear()
            raise IndexError("pop from empty list")

    pair._status_words[("cpu", 7)] = Taken([torch.ones(1, dtype=torch.int32)])
    word = pair._status("cpu")
    assert word.dtype == torch.int32 and word.tolist() == [0]
    assert pair._status("cpu").data_ptr() != word.data_ptr()


def test_status_words_of_threads_on_one_stream(one_stream):
    """Every call gets a word, a cleared one, and no two calls the same."""
    got, errors = [[] for _ in range(4)], []

    def take(mine):
        try:
            for _ in range(20_000):
                mine.append(pair._status("cpu"))
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        threads = [threading.Thread(target=take, args=(mine,)) for mine in got]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    assert errors == []
    words = [w for mine in got for w in mine]
    assert len({w.data_ptr() for w in words}) == 80_000
    assert int(torch.cat(words).abs().sum()) == 0


@pytest.fixture
def sizes_asked(monkeypatch):
    """paged_attention up to its workspace, without a device: what it asks the
    library for, and what it allocates."""
    asked, made = [], []
    pair._attention_workspace.cache_clear()

    class Native:
        @staticmethod
        def parts(device, *what):
            made.append(what)
            return tuple(torch.empty(0) for _ in what[::2])

    class Reached(Exception):
        pass

    def reached(*args, **kw):
        raise Reached

    def bytes_of(*sizes):
        asked.append((pair._device_index(), *sizes))
        return 1000 * (pair._device_index() + 1)

    monkeypatch.setattr(pair, "_native", lambda: Native)
    monkeypatch.setattr(pair, "pair_paged_attention_workspace_bytes", bytes_of)
    monkeypatch.setattr(pair, "_status", lambda device: None)
    monkeypatch.setattr(pair, "pair_paged_attention", reached)
    q, cache = torch.zeros(3, 4, 64), torch.zeros(2, 16, 2, 64)

    def call(max_q=1, max_len=20):
        with pytest.raises(Reached):
            pair.paged_attention(q, cache, cache, None, None, torch.zeros(3), max_q, max_len)
        return made[-1][-1]

    yield asked, call, monkeypatch
    pair._attention_workspace.cache_clear()


def test_workspaces_of_devices_are_apart(sizes_asked):
    """The workspace follows the device's compute units: another device's size is
    not taken from the first one's."""
    asked, call, patch = sizes_asked
    for device in (0, 1, 0, 1):
        patch.setattr(pair, "_device_index", lambda: device)
        assert call() == 1000 * (device + 1)
    assert [a[0] for a in asked] == [0, 1]               # each asked once


def test_workspaces_follow_the_bounds_values(sizes_asked):
    """Bounds given as tensors count by their value, not as the objects that they
    are: changed in place, they are other bounds."""
    asked, call, patch = sizes_asked
    patch.setattr(pair, "_device_index", lambda: 0)
    max_len = torch.tensor(20)
    call(max_len=max_len)
    max_len.fill_(4000)
    call(max_len=max_len)
    assert [a[-1] for a in asked] == [20, 4000] and all(type(a[-1]) is int for a in asked)
