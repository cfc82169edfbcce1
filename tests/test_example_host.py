"""What examples/decode.py refuses before it touches a device."""
import importlib.util
import os
import types

import pytest


@pytest.fixture(scope="module")
def decode():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")
    spec = importlib.util.spec_from_file_location("decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_bounded_cache_needs_normalised_heads(decode, monkeypatch, capsys):
    """Behind an eviction a token's place is not its position, and peqa_rope_append has no place."""
    with pytest.raises(ValueError, match="norms"):
        decode.generate(types.SimpleNamespace(norms=None), [[1, 2, 3]], 2, keep=8)
    monkeypatch.setattr("sys.argv", ["decode.py", "--keep", "64"])
    with pytest.raises(SystemExit) as e:
        decode.main()
    assert e.value.code == 2 and "--norms" in capsys.readouterr().err
