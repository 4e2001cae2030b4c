"""Build the HIP library libregioncache.so for gfx950 in-tree.

Every .hip source under csrc/ is compiled to an object with hipcc (in
parallel) and linked into a shared library next to this file.  The build
always recompiles; callers that only need the library load what exists.  A
build that fails leaves no library, and a library holds the digest of what it
was compiled from, so that one of other sources is not taken for these ones'.
"""
import concurrent.futures
import hashlib
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libregioncache.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "regioncache.h")
ARCH = "gfx950"


def hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
         # no packed-fp32 instruction selection (see the design notes)
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-result"]


def digest():
    """What rc_source_digest() of a library built now returns: SHA-256 of the
    flags and of every source's and header's name and content."""
    h = hashlib.sha256(repr(FLAGS).encode())
    for path in sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".hip", ".h"))) + [HEADER]:
        with open(path, "rb") as f:
            content = f.read()
        h.update(f"\n{os.path.basename(path)} {len(content)}\n".encode())
        h.update(content)
    return h.hexdigest()


def _compile(src, sources):
    obj = os.path.join(BUILD, os.path.basename(src)[:-4] + ".o")
    cmd = [hipcc()] + FLAGS + [f"-DRC_SOURCE_DIGEST={sources}", "-I", CSRC, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    if os.path.exists(LIB):
        os.remove(LIB)  # (processes that have it loaded keep it)
    sources = digest()
    srcs = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs, [sources] * len(srcs)))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    if digest() != sources:
        raise RuntimeError("a source changed while it was compiled: build again")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
