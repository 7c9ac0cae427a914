"""4-bit layers that no product could run are refused when they are made."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def S():
    from paper_2311_01305_amd import serving
    return serving


@pytest.fixture
def calls(S, monkeypatch):
    made = []
    monkeypatch.setattr(S.B, "aweq_quant_mx4", lambda *a, **k: made.append(a))
    return made


@pytest.mark.parametrize("N", [1, 2, 3, 5, 66])
def test_channels_that_are_no_multiple_of_four(S, calls, N):
    with pytest.raises(ValueError):
        S.Mx4Linear.from_weight(torch.zeros(N, 64))
    assert not calls


@pytest.mark.parametrize("N,K", [(0, 64), (8, 0), (8, 16), (8, 48), (8, 2 ** 20 + 32)])
def test_shapes_that_the_format_does_not_have(S, calls, N, K):
    with pytest.raises(ValueError):
        S.Mx4Linear.from_weight(torch.zeros(N, K))
    assert not calls


def test_biases_of_other_lengths_than_their_layers(S, calls):
    """Which together have as many values as the group has channels: they would go to other channels than their own."""
    K, Ns = 64, (8, 16)
    gb = types.SimpleNamespace(Ns=Ns, K=K, t={"inv_s": torch.ones(K), "status": None}, per=[{"W_hat": torch.zeros(N, K), "step_w": torch.zeros(N)} for N in Ns])
    for wrong in ([torch.ones(16), torch.ones(8)], [torch.ones(24), torch.ones(0)], [torch.ones(8), torch.ones(16).half()], [torch.ones(8), torch.ones(16, 1)]):
        with pytest.raises(ValueError):
            S.Mx4Linear.from_group(gb, biases=wrong)
    assert not calls
    right = S.Mx4Linear.from_group(gb, biases=[torch.ones(8), None])
    assert right.bias.tolist() == [1.0] * 8 + [0.0] * 16 and len(calls) == 1
