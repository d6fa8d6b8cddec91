"""CPU tests of what the build refuses: kernels that hold matrix operands in all registers, with some of them spilled."""
import os
import shutil

import pytest

from paper_2106_06899_amd import build

KERNELS = {"k_packed": "_ZN4topk12_GLOBAL__N_18k_packedILi64ELb1ELb1ELi2ELb1EEEvNS0_10PackedArgsE",
           "k_packed_dq": "_ZN4topk12_GLOBAL__N_111k_packed_dqILi64ELb1ELi2ELb0EEEvNS0_12BackwardArgsE",
           "k_packed_dkv": "_ZN4topk12_GLOBAL__N_112k_packed_dkvILi128ELb1ELb0EEEvNS0_12BackwardArgsE",
           "k_tree": "_ZN4topk12_GLOBAL__N_16k_treeILi128ELi9EEEvNS0_8TreeArgsE"}
OTHERS = {"k_tree_join": "_ZN4topk12_GLOBAL__N_111k_tree_joinILi64ELi1EEEvNS0_8TreeArgsE", "k_rows": "_ZN4topk6k_rowsItLi96ELi4ELi32EEEvNS_8RowsArgsE"}


def _log(spilled=()):
    lines = ["warning: something else"]
    for name, mangled in {**KERNELS, **OTHERS}.items():
        lines += [f"a.hip:1:1: remark: Function Name: {mangled} [-Rpass-analysis=kernel-resource-usage]", "    1 | __global__ void k()",
                  "a.hip:1:1: remark:     VGPRs: 256 [-Rpass-analysis=kernel-resource-usage]", "a.hip:1:1: remark:     SGPRs Spill: 9 [-Rpass-analysis=kernel-resource-usage]",
                  f"a.hip:1:1: remark:     VGPRs Spill: {7 if name in spilled else 0} [-Rpass-analysis=kernel-resource-usage]"]
    return "\n".join(lines)


def test_names_are_the_kernels():
    assert set(KERNELS) == set(build.NO_SPILLS)
    assert build.spills(_log()) == []


@pytest.mark.parametrize("name", sorted(KERNELS))
def test_spills_are_found(name):
    assert build.spills(_log([name])) == [f"{KERNELS[name]}: 7 vector registers spilled"]
    assert build.spills(_log().replace(KERNELS[name], "_Z5otherv")) == [f"{name}: not in the compiler's remarks"]


def test_other_kernels_may_spill():
    assert build.spills(_log(OTHERS)) == []


@pytest.mark.skipif(not shutil.which(build.HIPCC), reason="no compiler")
def test_the_compiler_says_so(tmp_path, monkeypatch):
    """A kernel of one of these names that needs more registers than there are is refused by the build, one that does not is
    built; a library that was there stays."""
    def source(n):
        return f"""#include <hip/hip_runtime.h>
namespace topk {{ namespace {{
template <int N> __global__ __launch_bounds__(1024) void k_tree(float* p) {{
  float x[N];
  for (int i = 0; i < N; ++i) x[i] = p[i * 1024 + threadIdx.x];
  __syncthreads();
  for (int j = 0; j < N; ++j) {{
    float s = 0;
    for (int i = 0; i < N; ++i) s += x[i] * x[(i * 7 + j) % N];
    p[j * 1024 + threadIdx.x] = s;
  }}
}} }}
void run(float* p) {{ k_tree<{n}><<<1, 1024>>>(p); }}
}}
"""
    out = str(tmp_path / "lib.so")
    monkeypatch.setattr(build, "NO_SPILLS", ("k_tree",))
    monkeypatch.setattr(build, "SOURCES", [str(tmp_path / "a.hip")])
    monkeypatch.setattr(build, "VARIANTS", {"main": (out, [])})
    (tmp_path / "a.hip").write_text(source(8))
    build.build(variants=("main",))
    before = os.path.getmtime(out)
    (tmp_path / "a.hip").write_text(source(160))
    with pytest.raises(RuntimeError, match="lib.so"):
        build.build(variants=("main",))
    assert os.path.getmtime(out) == before and not os.path.exists(out + ".tmp")
