"""Which kernels of the norms, the epilogue's backward pass and clipping keep values in scratch memory, by the built library's metadata (no GPU)."""
import os
import re
import subprocess

import pytest
import test_kernel_listing as K

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
pytestmark = [*K.pytestmark, pytest.mark.skipif(not os.path.exists(READELF), reason="no ROCm tools")]
KERNELS = ("rmsnorm_fwd_kernelI", "rmsnorm_bwd_kernelI", "act_bwd_kernelI", "column_sum_kernel", "grad_square_kernel", "grad_norm_kernel", "grad_scale_kernelI")
WIDE = ("rmsnorm_bwd_kernelILi16ELi2E", "rmsnorm_bwd_kernelILi16ELi4E")       # rows wider than 8192: known, and said beside the kernel


def test_only_the_backward_pass_of_wide_rows_uses_scratch_memory(tmp_path):
    scratch = {}
    with open(K.LIB, "rb") as f:
        data = f.read()
    for i, code in enumerate(K.code_objects(data)):
        path = tmp_path / f"code{i}.o"
        path.write_bytes(code)
        text = subprocess.run([READELF, "--notes", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
        names = re.findall(r"^\s+\.name:\s+(_Z\S+)$", text, re.M)
        sizes = [int(s) for s in re.findall(r"^\s+\.private_segment_fixed_size:\s+(\d+)$", text, re.M)]
        assert len(names) == len(sizes)
        scratch.update({n: s for n, s in zip(names, sizes) if any(k in n for k in KERNELS)})
    assert all(any(k in n for n in scratch) for k in (*KERNELS, *WIDE))
    assert {n: s for n, s in scratch.items() if s and not any(w in n for w in WIDE)} == {}
