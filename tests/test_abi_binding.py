"""The binding's own refusals (no GPU)."""
import subprocess

import pytest

from paper_2508_19078_amd import api


def test_a_library_that_lacks_entry_points_asks_for_a_build(tmp_path, monkeypatch):
    """A library of this ABI version built before an entry point was added."""
    src, so = tmp_path / "old.c", tmp_path / "old.so"
    src.write_text(f'int moe_abi_version(void) {{ return {api.ABI_VERSION}; }}\n'
                   'const char* moe_last_error(void) { return ""; }\n')
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    monkeypatch.setattr(api, "LIB_PATH", str(so))
    monkeypatch.setattr(api, "_lib", None)
    with pytest.raises(RuntimeError, match="rebuild it") as e:
        api.lib()
    assert "moe_route_topk" in str(e.value)            # the first that is missing


def test_an_older_version_is_named_before_its_symbols_are_looked_up(tmp_path, monkeypatch):
    src, so = tmp_path / "older.c", tmp_path / "older.so"
    src.write_text(f"int moe_abi_version(void) {{ return {api.ABI_VERSION - 1}; }}\n")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    monkeypatch.setattr(api, "LIB_PATH", str(so))
    monkeypatch.setattr(api, "_lib", None)
    with pytest.raises(RuntimeError, match=f"ABI version {api.ABI_VERSION - 1}.*rebuild it"):
        api.lib()


def test_norm_backward_without_any_row():
    with pytest.raises(ValueError, match="dS, dN, S and Y"):
        api.moe_sublayer_norm_bwd(None, None, None, None, None, None, None, None)
