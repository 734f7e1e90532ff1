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


@pytest.mark.parametrize("eps", [1e39, -1e39, float("inf"), float("nan")])
@pytest.mark.parametrize("call", ["join", "join_grad"])
def test_an_eps_that_is_no_number_of_fp32_is_refused(monkeypatch, call, eps):
    torch = pytest.importorskip("torch")
    import paper_2604_07239_amd as fa
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)  # the context's, as far as the binding can see
    c = object.__new__(fa.Fade)
    c.h, c.device, c.L = None, 0, fa.lib()
    x = torch.zeros((2, 8))
    with pytest.raises(fa.FadeError) as e:
        c.join(x, x, r=x, u=x, eps=eps) if call == "join" else c.join_grad(x, x, torch.zeros(4096), r=x, u=x, eps=eps)
    assert "eps" in str(e.value)
