"""Host side of the layer operators' torch functions (no GPU needed)."""
import types

from paper_2609_14706_amd import layer


def test_another_thread_during_the_first_call(monkeypatch):
    """The table of functions is empty or whole at every moment: a thread that
    finds it empty makes its own, one that finds it filled can use all of it."""
    seen = []

    class Library:
        def __getattr__(self, name):
            seen.append(len(layer._FN))
            return types.SimpleNamespace(name=name)
    monkeypatch.setattr(layer, "_FN", {})
    monkeypatch.setattr(layer, "load_library", Library)
    made = layer._library()
    assert len(seen) == len(made) == 10 and not any(seen)
    assert layer._library() is layer._FN and len(layer._FN) == 10
