"""Build of the CUDA library behind include/cllm.h (in-tree, sm_103a only).

``python -m paper_2403_00835_gb300.build`` compiles every ``csrc/*.cu`` with
nvcc for ``sm_103a`` in parallel and links ``_build/libcllm.so`` (CUDA runtime
linked statically, so the library loads on a machine without a GPU driver).
"""
from __future__ import annotations

import concurrent.futures as cf
import contextlib
import hashlib
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(OUT_DIR, "libcllm.so")


def _marshal_name() -> str:
    """Of the module built from csrc/marshal.cpp: it reads torch's and Python's objects as they lie in memory, so it
    serves the versions that it was built against, which its name tells."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch = "none"
    return f"_marshal-torch{torch}{sysconfig.get_config_var('EXT_SUFFIX') or '.so'}"


MARSHAL = os.path.join(OUT_DIR, _marshal_name())

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
              "-Xptxas", "-O3", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _fingerprint() -> str:
    h = hashlib.sha256()
    for d in (CSRC, INCLUDE):
        for f in sorted(os.listdir(d)):
            p = os.path.join(d, f)
            if os.path.isfile(p):
                h.update(f.encode())
                with open(p, "rb") as fh:
                    h.update(fh.read())
    h.update(" ".join(ARCH + NVCC_FLAGS).encode())
    return h.hexdigest()


def _build_marshal() -> None:
    """csrc/marshal.cpp against this interpreter's Python and torch; a note and no file if that fails (the
    next build tries again)."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return
    torch = spec.submodule_search_locations[0]
    lib = os.path.join(torch, "lib")
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-isystem", os.path.join(torch, "include"),
           "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "marshal.cpp"), "-o", tmp,
           "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cpu", "-lc10"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
        error = r.stderr[-500:] if r.returncode else ""
    except OSError as e:
        error = str(e)
    if error:
        print(f"{os.path.basename(MARSHAL)} not built, calls take their arguments in Python: {error}", file=sys.stderr)
    else:
        os.replace(tmp, MARSHAL)


def load_marshal():
    """The module built from csrc/marshal.cpp, or None: not built, or, with a note, not one that this interpreter loads."""
    if not os.path.exists(MARSHAL):
        return None
    try:
        spec = importlib.util.spec_from_file_location("_marshal", MARSHAL)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except Exception as e:  # (a damaged file, a symbol that torch lacks)
        print(f"{os.path.basename(MARSHAL)} not loaded, calls take their arguments in Python: {e}", file=sys.stderr)
        return None
    return module


def build(force: bool = False, verbose: bool = False, extra_flags=None) -> str:
    """Compile the library if sources changed; returns the .so path."""
    os.makedirs(OUT_DIR, exist_ok=True)
    stamp = os.path.join(OUT_DIR, "stamp")
    fp = _fingerprint() + " ".join(extra_flags or [])
    if not force and os.path.exists(LIB) and os.path.exists(stamp):
        with open(stamp) as fh:
            if fh.read() == fp:
                if not os.path.exists(MARSHAL):  # (another interpreter or torch, or it failed)
                    _build_marshal()
                return LIB
    nvcc = _nvcc()
    flags = NVCC_FLAGS + list(extra_flags or [])
    for f in os.listdir(OUT_DIR):
        # of the sources before, whoever they were built for (.tmp: another process is at it)
        if f.startswith("_marshal") and ".tmp" not in f:
            with contextlib.suppress(FileNotFoundError):
                os.remove(os.path.join(OUT_DIR, f))

    def compile_one(src):
        obj = os.path.join(OUT_DIR, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc] + ARCH + flags + ["-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr, file=sys.stderr)
        return obj

    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs) + 1, os.cpu_count() or 4)) as ex:
        marshal = ex.submit(_build_marshal)
        objs = list(ex.map(compile_one, srcs))
        marshal.result()
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc] + ARCH + ["-shared", "-o", tmp] + objs + ["-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    with open(stamp, "w") as fh:
        fh.write(fp)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
