"""The library's sources and what is built of them."""
import concurrent.futures
import os
import subprocess

import pytest

from paper_2608_29809_amd import build

SOURCES = sorted(f for f in os.listdir(build.CSRC) if f.endswith(".hip"))


def has_hipcc():
    try:
        build.hipcc()
    except RuntimeError:
        return False
    return True


needs_hipcc = pytest.mark.skipif(not has_hipcc(), reason="needs hipcc")


@needs_hipcc
def test_sources_compile():
    """Every source is accepted as the build compiles it, for the host and for the GPU (template bodies and launch bounds among it)."""
    def errors(name):
        cmd = [build.hipcc()] + build.FLAGS + ["-I", build.CSRC, "-fsyntax-only", os.path.join(build.CSRC, name)]
        r = subprocess.run(cmd, capture_output=True, text=True)
        return [line for line in r.stderr.splitlines() if "error" in line][:3] or ["failed"] if r.returncode else None

    with concurrent.futures.ThreadPoolExecutor(max_workers=4) as ex:
        failed = {n: e for n, e in zip(SOURCES, ex.map(errors, SOURCES)) if e}
    assert not failed, failed
