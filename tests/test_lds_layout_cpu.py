"""Where the join of beam search's lists keeps its entries in LDS: behind its own arrays, at the alignment of what lies
there."""

import os
import re
import subprocess

from paper_2606_26587_amd import build as B


def test_candidates_lie_at_their_alignment(tmp_path):
    out = str(tmp_path / "beam.s")
    flags = [f for f in B.HIP_FLAGS if f != "-O3"] + ["-O1"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(B.CSRC, "sharq_beam.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    sizes = re.findall(r"\.group_segment_fixed_size:\s*(\d+).*?\.name:\s*(\S+)", text, re.S)
    size = {name: int(n) for n, name in sizes}
    picks = [n for n in size if "k_beam_pick" in n]
    assert len(picks) == 1
    # BeamKey holds 16 bytes and is read as such; what the launch adds begins here
    assert size[picks[0]] % 16 == 0
