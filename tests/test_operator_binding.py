"""The binding's handling of arguments where no device is needed."""
import pytest


def test_first_calls_of_two_threads_find_every_type(monkeypatch):
    """A thread that comes while another one fills the tables of types has its tokens accepted."""
    torch = pytest.importorskip("torch")
    from paper_2604_07239_amd import binding
    tokens, seen = torch.zeros(1, dtype=torch.uint8), []

    class Filling(dict):
        def update(self, *args):
            super().update(*args)
            seen.append(binding._late_type(binding._TOKENS, tokens))  # what that thread would see

    monkeypatch.setattr(binding, "_TYPES", Filling())
    monkeypatch.setattr(binding, "_TOKENS", {})
    assert binding._late_type(binding._TYPES, torch.zeros(1)) == binding.F32
    assert seen == [binding.TOKEN_U8]
