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
