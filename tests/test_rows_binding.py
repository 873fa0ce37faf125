"""The binding of the operators on logits rows (CPU): what several threads share
on first use."""
import pytest

torch = pytest.importorskip("torch")


def test_types_are_whole_whenever_they_are_seen(monkeypatch):
    """A thread that finds the table of types filled finds all of it."""
    from paper_2606_00722_amd import epic

    seen = []

    class Watched(dict):
        def update(self, *a, **kw):
            super().update(*a, **kw)
            seen.append(set(self))

        def __setitem__(self, k, v):
            super().__setitem__(k, v)
            seen.append(set(self))

    monkeypatch.setattr(epic, "_DTYPES", Watched())
    monkeypatch.setattr(epic, "_torch", None)
    table = epic._dtypes()
    assert table[torch.float32] == 0 and table["i32"] is torch.int32 and epic._torch is torch
    assert seen and all(keys == set(table) for keys in seen)
