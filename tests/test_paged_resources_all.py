"""Scratch memory of every kernel on a paged cache, both storage types, as the compiler reports it for gfx950 (no GPU needed)."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2601_07353_amd import build as B

# source -> kernels
SOURCES = {"paged_rows.hip": 6}
for _t in ("bf16", "f16"):
    SOURCES.update({"paged_attention_%s_far.hip" % _t: 19, "paged_weights_%s.hip" % _t: 24, "paged_attention_%s_64.hip" % _t: 13,
                    "paged_attention_%s_128.hip" % _t: 13, "paged_attention_%s_256.hip" % _t: 9})

# (head width, wavefronts, capped) -> bytes a lane, of many rows' tiles whose scores fall with the distance; all others have none
DISTANCE = {(128, 4, 0): 100, (128, 4, 1): 80, (128, 8, 0): 96, (128, 8, 1): 92, (256, 4, 0): 52, (256, 4, 1): 84}


def test_scratch_memory_of_every_kernel():
    def one(source):
        return subprocess.run([B._hipcc(), *B.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S",
                               os.path.join(B.CSRC, source), "-o", os.devnull], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, check=True).stdout
    assert set(SOURCES) == {s for s in B.SOURCES if s.startswith("paged_") and s != "paged_api.hip"}
    with ThreadPoolExecutor(max_workers=6) as ex:
        said = dict(zip(SOURCES, ex.map(one, SOURCES)))
    for source, kernels in SOURCES.items():
        found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", said[source], re.S)
        assert len(found) == kernels, (source, len(found))
        for name, size in found:
            m = re.search(r"paged_attention_kernelILb[01]ELi(\d+)ELi([48])ELb([01])ELb1E", name)
            assert int(size) <= (DISTANCE.get(tuple(int(x) for x in m.groups()), 0) if m else 0), (name, size)
