"""What the compiler makes of the paged cache's kernels where no result would show a loss (no GPU)."""
import re

import pytest

from test_kernel_build_host import _device_code


@pytest.mark.parametrize("source,kernels", [("fkv_decode_quant.hip", 4), ("fkv_append.hip", 7)])
def test_nothing_goes_to_scratch(source, kernels, tmp_path):
    """Neither registers nor a copy of the arguments, which an index that differs between lanes can cause."""
    said = _device_code(source, tmp_path, "-c", "-Rpass-analysis=kernel-resource-usage")[1]
    names = re.findall(r"Function Name: (\S+)", said)
    scratch = [int(n) for n in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", said)]
    assert len(names) == len(scratch) == kernels and not any(scratch), list(zip(names, scratch))


def test_a_tile_is_nine_loads(tmp_path):
    """The decode kernel's waits count loads: the queries' 2, then 9 of each tile, scales and K ahead of V, and nothing else between them."""
    out = _device_code("fkv_decode_quant.hip", tmp_path, "-S")[0]
    bodies = re.findall(r"^_Z\w*k_decode_quant\w*:(.*?)^\.Lfunc_end", open(out).read(), re.S | re.M)
    assert len(bodies) == 4
    for body in bodies:
        runs, run = [], ""
        for line in (l.strip() for l in body.splitlines()):
            if line.startswith((".LBB", "s_cbranch", "s_branch", "s_waitcnt vmcnt")):
                runs.append(run)
                run = ""
            elif line.startswith("buffer_load_dwordx4") and "lds" in line:
                run += "q"
            elif line.startswith("global_load_lds_dwordx4"):
                run += "t"
            elif line.startswith("global_load_lds_dword "):
                run += "s"
            elif line.startswith(("global_load", "flat_load", "buffer_load")):
                run += "?"
        queries = [r.replace("?", "") for r in runs if "q" in r]  # the page entries may be asked for beside them
        assert queries == ["qq"], runs
        tiles = [r for r in runs if set(r) & set("ts")]
        assert sorted(set(tiles)) == ["stttt", "stttttttt", "tttt"], tiles  # a wave's first two tiles; in the loop K and V by themselves
