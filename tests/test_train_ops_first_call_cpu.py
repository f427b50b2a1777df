"""The first call of a training-step operator, from several host threads at once."""
import threading

import pytest

from paper_2606_27216_amd import train_ops as ops


@pytest.mark.parametrize("table", ["_INDEX", "_TYPES"])
def test_a_thread_that_comes_in_between_finds_everything_or_fills_it_in(monkeypatch, table):
    """A second thread makes its first call at the moment at which the first one has just
    filled one of the tables: whatever it then uses is there."""
    pytest.importorskip("torch")
    seen = []

    def second():
        ops._torch()
        seen.append((ops._device, ops._raw_stream, len(ops._TYPES), len(ops._INDEX)))

    class Table(dict):
        def update(self, *args):
            dict.update(self, *args)
            if not seen:
                seen.append(None)
                t = threading.Thread(target=second)
                t.start()
                t.join()

    for name, empty in (("_INDEX", {}), ("_TYPES", {}), ("_device", None), ("_raw_stream", None)):
        monkeypatch.setattr(ops, name, Table() if name == table else empty)
    ops._torch()
    device, raw_stream, types, indexes = seen[1]
    assert callable(device) and callable(raw_stream) and types == 2 and indexes == 2
