"""The kernels over the vocabulary keep everything in registers: no scratch memory, and vector registers for the wavefronts that keep the
memory busy (six on a SIMD of 512 registers a lane where 16-byte pieces hold eight logits, five where they hold four)."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2605_27081_amd import build as libbuild


@pytest.mark.parametrize("src,kernel,most", [("head.hip", r"head_scan_kernelILi\d+ELi1E", 80), ("head.hip", r"head_scan_kernelILi\d+ELi0E", 96),
                                             ("head.hip", "head_join_kernel", 128), ("head_grad.hip", "head_grad_kernel", 80)])
def test_no_scratch_and_room_for_wavefronts(src, kernel, most):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "k.s")
        flags = [f for f in libbuild.FLAGS if f != "-fPIC"]
        r = subprocess.run([libbuild.HIPCC, *flags, "-S", "--cuda-device-only", os.path.join(libbuild.CSRC, src), "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        text = open(out).read()
    bodies = [(n, b) for n, b in re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", text, re.S) if re.search(kernel, n)]
    assert bodies
    for n, body in bodies:
        assert int(re.search(r"\.amdhsa_next_free_vgpr (\d+)", body).group(1)) <= most, n
        assert int(re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", body).group(1)) == 0, n
