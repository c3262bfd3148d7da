"""The attention layer's command refuses sizes that it cannot run, a chunk of no tokens among them, which would never
read its prompts (no device needed)."""
import pytest

pytest.importorskip("torch")

from paper_2406_20037_amd import attn8  # noqa: E402


@pytest.mark.parametrize("name, value", [("chunk", 0), ("chunk", -5), ("seqs", 0), ("prompt", -1), ("tokens", -1), ("window", -1),
                                         ("width", 0), ("heads", 0), ("kv-heads", 0), ("dim", 0)])
def test_sizes(name, value, capsys):
    with pytest.raises(SystemExit) as e:
        attn8.main([f"--{name}", str(value)])
    assert e.value.code == 2 and f"--{name} {value}" in capsys.readouterr().err
