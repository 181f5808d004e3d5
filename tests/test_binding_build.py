"""The compiled binding belongs to one Python and one torch: built for others it is built again, and not loaded before that."""
import pytest


@pytest.fixture()
def built():
    from paper_2605_31035_gb300 import build
    build.build()
    return build


def test_stamp_is_this_python_and_torch(built):
    import sysconfig

    import torch
    text = open(built.BINDING_ABI).read()
    assert torch.__version__ in text and sysconfig.get_config_var("SOABI") in text
    assert built.binding_fits() and built.up_to_date()


@pytest.mark.parametrize("stamp", [None, "", "cpython-39 torch 1.0 cxx11 0\n"])
def test_a_binding_for_others_is_stale(built, stamp, tmp_path, monkeypatch):
    from paper_2605_31035_gb300 import ops
    other = tmp_path / "_binding.abi"
    if stamp is not None:
        other.write_text(stamp)
    monkeypatch.setattr(built, "BINDING_ABI", str(other))
    assert not built.up_to_date()
    monkeypatch.setattr(ops, "_binding", None)
    with pytest.raises(RuntimeError, match="built for"):
        ops._native()


def test_another_torch_is_noticed(built, monkeypatch):
    import torch
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".other")
    assert not built.up_to_date()


def test_linking_stamps(built, tmp_path, monkeypatch):
    """A link replaces both files, and a failed one leaves the stamp's module in place."""
    import os
    target, stamp = tmp_path / "_binding.so", tmp_path / "_binding.abi"
    monkeypatch.setattr(built, "BINDING", str(target))
    monkeypatch.setattr(built, "BINDING_ABI", str(stamp))
    stamp.write_text("old\n")
    with pytest.raises(RuntimeError, match="link"):
        built._link_binding(str(tmp_path / "none.o"))
    assert stamp.read_text() == "old\n" and not target.exists()
    built._link_binding(os.path.join(built.BUILD, "binding.o"))
    assert target.exists() and stamp.read_text() == built.abi()
    assert sorted(p.name for p in tmp_path.iterdir()) == ["_binding.abi", "_binding.so"]
