"""The library's sources and what is built of them."""
import concurrent.futures
import os
import subprocess

import pytest

from paper_2608_29809_amd import abi, build

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


def test_library_is_of_these_sources():
    assert abi.LIB.rc_source_digest().decode() == build.digest()


def test_library_of_other_sources_is_refused(monkeypatch):
    monkeypatch.setattr(build, "digest", lambda: "0" * 64)
    with pytest.raises(ImportError, match="other sources"):
        abi._load()


def test_digest_sees_every_source(monkeypatch, tmp_path):
    """One byte more, another name or another flag is another digest; other files do not count."""
    monkeypatch.setattr(build, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(build, "HEADER", str(tmp_path / "api.h"))
    (tmp_path / "csrc").mkdir()
    a, b, api = tmp_path / "csrc" / "a.hip", tmp_path / "csrc" / "b.h", tmp_path / "api.h"
    for f in (a, b, api):
        f.write_text("int x;\n")
    seen = [build.digest()]
    (tmp_path / "csrc" / "notes.txt").write_text("x")
    assert build.digest() == seen[0]
    for f in (a, b, api):
        f.write_text("int x; \n")
        seen.append(build.digest())
    b.rename(tmp_path / "csrc" / "c.h")
    seen.append(build.digest())
    monkeypatch.setattr(build, "FLAGS", build.FLAGS + ["-g"])
    seen.append(build.digest())
    assert len(set(seen)) == len(seen)


@pytest.mark.parametrize("fails", ["compile", "link", "edit"])
def test_failed_build_leaves_no_library(monkeypatch, tmp_path, fails):
    """The library of an earlier build does not stand for sources that were not built."""
    for name in ("BUILD", "LIB", "CSRC", "HEADER"):
        monkeypatch.setattr(build, name, str(tmp_path / name.lower()))
    os.mkdir(build.CSRC)
    source = tmp_path / "csrc" / "a.hip"
    source.write_text("int x;\n")
    (tmp_path / "header").write_text("")
    (tmp_path / "lib").write_text("an earlier library")
    compiler = tmp_path / "compiler"
    compiler.write_text({"compile": "#!/bin/sh\nexit 1\n",
                         "link": '#!/bin/sh\ntest "$1" != -shared\n',
                         "edit": f'#!/bin/sh\nif test "$1" = -shared; then echo "int y;" > {source}; echo > {build.LIB}.tmp; fi\n'}[fails])
    compiler.chmod(0o755)
    monkeypatch.setattr(build, "hipcc", lambda: str(compiler))
    with pytest.raises(RuntimeError):
        build.build()
    assert not os.path.exists(build.LIB)


@pytest.mark.parametrize("part", ["CSRC", "HEADER"])
def test_library_without_its_sources_is_loaded(monkeypatch, tmp_path, part):
    monkeypatch.setattr(build, part, str(tmp_path / "missing"))
    assert abi._load().rc_source_digest()
