"""The package's names are the binding's, at every use (no device needed)."""
import subprocess
import sys

import pytest

import paper_2406_20037_amd as ds


@pytest.mark.parametrize("name", ["kernel_run", "ds_q8_matmul", "Q8"])
def test_a_replaced_name_is_seen(monkeypatch, name):
    before = getattr(ds, name)
    assert before is getattr(ds._lib, name)
    other = object()
    monkeypatch.setattr(ds._lib, name, other)
    assert getattr(ds, name) is other
    monkeypatch.undo()
    assert getattr(ds, name) is before


def test_unknown_names():
    with pytest.raises(AttributeError):
        ds.no_such_name
    assert all(hasattr(ds, name) for name in ds.__all__)


def test_the_binding_is_loaded_on_first_use():
    code = ("import sys, paper_2406_20037_amd as ds; n = 'paper_2406_20037_amd._lib'; assert n not in sys.modules; "
            "ds.kernel_run; assert n in sys.modules and ds._lib is sys.modules[n]")
    subprocess.run([sys.executable, "-c", code], check=True)
