"""Registers of the kernels on a paged cache, as the compiler reports them for gfx950 (no GPU needed)."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2601_07353_amd import build as B

SOURCES = {"paged_rows.hip": 6, "paged_weights_bf16.hip": 24, "paged_attention_bf16_64.hip": 13, "paged_attention_bf16_128.hip": 13, "paged_attention_f16_256.hip": 9}


def test_kernels_do_not_spill():
    """No scratch memory, but for tiles of many rows whose scores fall with the distance (some registers that the loop over tiles
    reads back once a tile)."""
    def one(source):
        return subprocess.run([B._hipcc(), *B.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S",
                               os.path.join(B.CSRC, source), "-o", os.devnull], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, check=True).stdout
    with ThreadPoolExecutor(max_workers=5) as ex:
        said = dict(zip(SOURCES, ex.map(one, SOURCES)))
    for source, kernels in SOURCES.items():
        found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", said[source], re.S)
        assert len(found) == kernels, (source, len(found))
        for name, size in found:
            distance = re.search(r"paged_attention_kernelILb[01]ELi(128|256)ELi[48]ELb[01]ELb1E", name)
            assert int(size) <= (128 if distance else 0), (name, size)
