"""The command that calibrates a block, runs a shared prompt and decodes a batch behind it."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix", [0, 1, 70])
def test_command(capsys, prefix):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import serving
    serving.main(["--hidden", "256", "--heads", "2", "--key-heads", "1", "--prefix", str(prefix), "--batch", "3", "--steps", "4", "--codes"])
    out = capsys.readouterr().out
    assert f"behind {prefix} shared tokens" in out and "status 0" in out
