"""CPU-only: the window attention kernels load their tiles through inline assembly (test_isa_hazards.py says what that asks for): nothing is in
flight at a barrier that publishes a tile or at the end, and no assembly block loads into registers."""
import os

from test_isa_hazards import ROOT, _assembly, scan

CSRC = os.path.join(ROOT, "paper_2204_06514_amd", "csrc")


def test_window_tile_loads_are_waited_for(tmp_path):
    for name, kernels in (("kernels_window_mfma.hip", 40), ("kernels_window_dkv.hip", 5)):
        text = _assembly(tmp_path, os.path.join(CSRC, name), ("-mllvm", "-amdgpu-mfma-vgpr-form=1"))  # options as in build.py
        n, bad = scan(text.replace("window_", "attn_window_"), r"_ZN3fax\d+attn_window_\w+")  # none allowed in flight
        assert n >= kernels, (name, n)
        assert not bad, {k: v[:3] for k, v in bad.items()}


def test_wide_tile_loads_are_waited_for(tmp_path):
    text = _assembly(tmp_path, os.path.join(CSRC, "kernels_window_wide.hip"), ())
    n, bad = scan(text.replace("window_", "attn_window_"), r"_ZN3fax\d+attn_window_\w+")
    assert n >= 4, n
    assert not bad, {k: v[:3] for k, v in bad.items()}
