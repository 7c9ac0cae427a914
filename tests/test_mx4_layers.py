"""4-bit layers that no product could run are refused when they are made."""
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
