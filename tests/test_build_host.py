"""The build's second product, the native marshalling, is made again whenever it is missing, of another PyTorch or
failed before; the library beside it is left alone then."""
import os
import sysconfig

import pytest


@pytest.fixture
def B(monkeypatch, tmp_path):
    from paper_2609_15359_gb300 import build
    build.build()
    if not build.marshal_up_to_date():
        pytest.skip("PyTorch's headers do not compile here")
    assert os.path.basename(build.MARSHAL) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / os.path.basename(build.MARSHAL)))
    monkeypatch.setattr(build, "PKG", str(tmp_path))  # a module of the old name would lie there
    monkeypatch.setattr(build, "_marshal_key", lambda: str(tmp_path / "key"))
    return build


def test_the_module_is_made_alone_and_again(B, tmp_path, monkeypatch, capsys):
    at = os.path.getmtime(B.LIB)
    (tmp_path / "_marshal.so").write_bytes(b"of any Python")
    assert B.library_up_to_date() and not B.up_to_date()
    B.build()
    assert B.up_to_date() and os.path.getmtime(B.LIB) == at and not (tmp_path / "_marshal.so").exists()
    made = os.path.getmtime(B.MARSHAL)
    B.build()
    assert os.path.getmtime(B.MARSHAL) == made  # nothing to do
    with monkeypatch.context() as m:  # another PyTorch, whose headers are missing
        m.setattr(B, "torch_version", lambda: "99.0")
        m.setattr(B, "_torch_root", lambda: str(tmp_path))
        assert not B.up_to_date()
        B.build()
        assert "marshalled in Python" in capsys.readouterr().err and not os.path.exists(B.MARSHAL) and not B.up_to_date()
    assert not B.up_to_date()
    B.build()  # and found again
    assert B.up_to_date() and os.path.getmtime(B.LIB) == at


def test_a_module_of_another_pytorch_is_not_up_to_date(B, tmp_path, monkeypatch):
    B.build()
    assert B.up_to_date()
    (tmp_path / "key").write_text("1.0")
    assert not B.up_to_date()
