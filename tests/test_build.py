"""The join's parts build without the attention operators' binding."""
import os

import pytest

import __graft_entry__ as entry
from oracle import oracle
from paper_2609_11938_amd import attn, build


def test_the_join_is_built_where_the_binding_cannot_be(monkeypatch):
    done = []

    def run(cmd, out, verbose):
        if out == build.BIND:
            raise RuntimeError("no C++ compiler for torch's headers")
        done.append(out)

    monkeypatch.setattr(build, "_run", run)
    monkeypatch.setattr(oracle, "build", lambda: done.append(oracle.LIB))
    with pytest.raises(RuntimeError):
        entry.build()
    assert done == [build.LIB, oracle.LIB]


def test_smoke_of_the_join_does_not_wait_for_the_binding(monkeypatch, tmp_path):
    from paper_2609_11938_amd import opattr

    there = tmp_path / "built.so"
    there.write_bytes(b"")
    monkeypatch.setattr(opattr, "LIB_PATH", str(there))
    monkeypatch.setattr(oracle, "LIB", str(there))
    monkeypatch.setattr(attn, "BIND_PATH", os.path.join(str(tmp_path), "missing.so"))
    monkeypatch.setattr(entry, "build", lambda: pytest.fail("built again"))
    entry._ensure_built()


@pytest.mark.parametrize("abi", [False, True])
def test_the_binding_is_compiled_with_torchs_abi(monkeypatch, abi):
    import torch

    cmds = []
    monkeypatch.setattr(build, "_run", lambda cmd, out, verbose: cmds.append(cmd))
    monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: abi)
    build.build_binding()
    assert f"-D_GLIBCXX_USE_CXX11_ABI={int(abi)}" in cmds[0]
