"""The sizes that the attention over a shared prefix refuses, and their workspaces: nothing here needs a GPU."""
import pytest

P = 0x10000  # a fake, 16-byte aligned, never dereferenced "device pointer"


@pytest.fixture(scope="module")
def B():
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def call(lib, **changed):
    c = dict(T=64, Hq=8, Hk=2, D=128, B=64, max_q=1, prefix_len=100, max_len=5000, scale=0.1, pages=64)
    c.update(changed)
    width = c["Hq"] * c["D"]
    sizes = (c["T"], c["Hq"], c["Hk"], c["D"], c["B"], c["max_q"], c["prefix_len"], c["max_len"])
    # (no workspace where some is needed: what is not refused for its shape is refused for that)
    with pytest.raises(lib.AweqError) as e:
        lib.aweq_prefix_attention(P, lib.AWEQ_F16, c["T"], c["Hq"], c["D"], width, P, P, None, None, lib.AWEQ_F16, c["pages"], 16, c["Hk"], P, c["prefix_len"], P, 400, P, P, c["B"],
                                c["max_len"], c["max_q"], c["scale"], P, width, None, None, ws_bytes=0, stream=0)
    return e.value.name, lib.aweq_prefix_attention_ws(*sizes), lib.aweq_prefix_attention_ws_most(*sizes)


def test_sizes_up_to_the_limits(B):
    for inside in (dict(), dict(T=2097151, B=1, max_q=4096, max_len=20000), dict(T=255, Hq=65536, Hk=8192, B=255), dict(B=1 << 20, T=1 << 20, Hk=1),
                   dict(prefix_len=1 << 29), dict(max_len=1 << 29), dict(pages=0x7fffffff)):
        name, need, most = call(B, **inside)
        assert name == "AWEQ_ERR_WORKSPACE" and 0 < need <= most, inside


def test_sizes_beyond_them(B):
    for beyond in (dict(T=2097152, B=1, max_q=4096), dict(T=1 << 24, Hq=1, Hk=1, B=1, max_q=1 << 24), dict(T=256, Hq=65536, Hk=8192), dict(T=2, B=2, Hq=65544, Hk=8),
                   dict(B=(1 << 20) + 1, T=1 << 20), dict(B=1 << 20, Hk=32, Hq=32, T=1 << 18), dict(prefix_len=(1 << 29) + 1), dict(max_len=(1 << 29) + 1)):
        assert call(B, **beyond) == ("AWEQ_ERR_SHAPE", 0, 0), beyond
    assert call(B, pages=0x80000000)[0] == "AWEQ_ERR_SHAPE"


def test_scales(B):
    """To base 2 they have to be finite."""
    assert call(B, scale=1.6e38)[0] == "AWEQ_ERR_WORKSPACE"
    for scale in (1.8e38, 3e38, float("inf"), float("nan"), 0.0, -1.0):
        assert call(B, scale=scale)[0] == "AWEQ_ERR_SHAPE"
