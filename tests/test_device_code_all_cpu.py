"""The other device sources read as test_device_code_cpu.py reads the state cache
and the parameter lists: no select or branch takes a carry for a comparison."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2508_06993_amd.build import COMMON_FLAGS, DEVICE_FLAGS, hipcc, sources
from test_device_code_cpu import flags_misread

READ_THERE = ("state_cache.hip", "params.hip")


def test_no_flag_is_misread_in_any_source(tmp_path):
    flags = [f for f in COMMON_FLAGS if f != "-fPIC"]

    def read(source):
        out = str(tmp_path / (os.path.basename(source) + ".s"))
        subprocess.run([hipcc(), *flags, *DEVICE_FLAGS, "-S", "--cuda-device-only", source, "-o", out],
                       check=True, capture_output=True)
        with open(out) as f:
            return f.read()
    files = [s for s in sources() if os.path.basename(s) not in READ_THERE]
    with ThreadPoolExecutor(8) as pool:
        texts = list(pool.map(read, files))
    assert sum(t.count("s_endpgm") for t in texts) > 50
    for source, text in zip(files, texts):
        assert flags_misread(text) == [], os.path.basename(source)
