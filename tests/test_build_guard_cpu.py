"""What the build refuses by the compiler's remarks, here made up: kernels in scratch memory, and spilled registers but for those that are allowed by name."""
from __future__ import annotations

import os

import pytest

from paper_2609_24875_amd import build as B


def _compiled(monkeypatch, tmp_path, kernels):
    """_compile with remarks that say this of the kernels: {name: (scratch bytes, spilled registers)}."""
    said = "".join(f"a.hip:1:1: remark: Function Name: {k} [-R]\na.hip:1:1: remark:     ScratchSize [bytes/lane]: {s} [-R]\n"
                   f"a.hip:1:1: remark:     SGPRs Spill: 9 [-R]\na.hip:1:1: remark:     VGPRs Spill: {v} [-R]\n" for k, (s, v) in kernels.items())

    def run(cmd):
        out = cmd[cmd.index("-o") + 1]
        with open(out, "w") as f:
            f.write("made")
        return said if "-c" in cmd else ""
    monkeypatch.setattr(B, "_run", run)
    monkeypatch.setattr(B, "hipcc", lambda: "hipcc")
    out = str(tmp_path / "lib.so")
    try:
        return B._compile(["a.hip"], out, False) == out and os.path.exists(out)
    finally:
        assert not os.path.exists(out + ".tmp")


ALLOWED = "_ZN12_GLOBAL__N_113k_attn_sharedILi192ELi8ELi1ELb1ELi2EEEvNS_10SharedArgsE"


@pytest.mark.parametrize("name", ["_Z11k_gemm_wideILi1EEv", "_Z6k_ropeIfEv", "_Z11k_kv_appendv", "_Z6k_attnILi128ELi16ELi1EEv", "_Z14k_weights_manyILi192ELi8EEv",
                                  "_Z14k_evict_choosev", "k_attn_sharedILi128ELi8ELi1ELb1ELi2EE", "k_attn_sharedILi192ELi4ELi1ELb1ELi2EE",
                                  "k_attn_sharedILi192ELi16ELi1ELb1ELi2EE"])
@pytest.mark.parametrize("scratch,spill", [(0, 1), (0, 4), (0, 5), (4, 0), (64, 16)])
def test_spills_and_scratch_are_refused(monkeypatch, tmp_path, name, scratch, spill):
    with pytest.raises(RuntimeError, match=name):
        _compiled(monkeypatch, tmp_path, {"_Z5k_fitv": (0, 0), name: (scratch, spill)})


def test_what_is_allowed(monkeypatch, tmp_path):
    assert _compiled(monkeypatch, tmp_path, {"_Z11k_gemm_wideILi1EEv": (0, 0), ALLOWED: (0, 3), "_Z8k_searchv": (128, 20)})


@pytest.mark.parametrize("scratch,spill", [(4, 0), (4, 3), (0, 4)])
def test_what_is_allowed_has_a_bound(monkeypatch, tmp_path, scratch, spill):
    with pytest.raises(RuntimeError, match="k_attn_shared"):
        _compiled(monkeypatch, tmp_path, {ALLOWED: (scratch, spill)})
