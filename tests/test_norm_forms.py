"""Which forms of the norm's kernels the library holds: those that a width of up to 16384 reaches, and no others.  No GPU needed."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2206_03382_amd import moe


@pytest.mark.skipif(shutil.which("nm") is None or not os.path.exists(moe.LIB_PATH), reason="needs the built library and nm")
@pytest.mark.parametrize("kernel", ["rms_norm_kernel", "rms_norm_backward_kernel"])
def test_forms_are_reached(kernel):
    names = subprocess.run(["nm", "-C", moe.LIB_PATH], capture_output=True, text=True, check=True).stdout
    held = {(t, int(lanes), int(pieces)) for t, lanes, pieces in re.findall(r"\b" + kernel + r"<(unsigned short|float), (\d+), (\d+)>", names)}
    assert held
    for t, lanes, pieces in held:
        most = 16384 // (8 if t == "unsigned short" else 4)        # 16-byte pieces of the widest row
        least = {64: 0, 256: 64, 1024: 1024}[lanes]                # rows of fewer take fewer lanes
        per_lane = [-(-p // lanes) for p in range(least + 1, min(most, {64: 128, 256: 1024, 1024: 1 << 30}[lanes]) + 1)]
        below = max([0] + [p for u, q, p in held if (u, q) == (t, lanes) and p < pieces])
        assert any(below < n <= pieces for n in per_lane), f"no width reaches {kernel}<{t}, {lanes}, {pieces}>"
