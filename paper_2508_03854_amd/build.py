"""Builds libtbe355.so (gfx950 only) next to this file with hipcc.  No JIT: the library is built ahead of
time, in-tree, and loaded by binding.py."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtbe355.so")
SOURCES = ["tbe_api.hip", "tbe_forward.hip", "tbe_sort.hip", "tbe_sort_small.hip", "tbe_lists.hip", "tbe_dense.hip", "tbe_backward.hip", "tbe_sync.hip", "tbe_norm.hip", "tbe_attention.hip", "tbe_attention_backward.hip", "tbe_encoder_api.hip", "tbe_calibrate.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _newer(target: str, deps) -> bool:
    if not os.path.exists(target):
        return False
    t = os.path.getmtime(target)
    return all(os.path.getmtime(d) <= t for d in deps)


def source_digest() -> str:
    """Twelve hex digits that name the sources a library is built from; the library reports them
    through tbe_build_info(), and a counter profile records them, so that measured traffic is only ever attached to
    the kernels it was measured on."""
    import hashlib
    hsh = hashlib.sha256()
    files = sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".hip")))
    files.append(os.path.join(ROOT, "include", "tbe355.h"))
    for f in files:
        hsh.update(os.path.basename(f).encode())
        hsh.update(open(f, "rb").read())
    return hsh.hexdigest()[:12]


def build(force: bool = True, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    headers.append(os.path.join(ROOT, "include", "tbe355.h"))
    digest = source_digest()

    def compile_one(src: str) -> str:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".hip", ".o"))
        deps = [s] + headers
        if src == "tbe_api.hip":   # carries the digest of all sources
            deps = deps + [os.path.join(CSRC, f) for f in SOURCES]
        if force or not _newer(o, deps):
            cmd = [HIPCC] + FLAGS + ["-c", s, "-o", o]
            if src == "tbe_api.hip":
                cmd.insert(-4, '-DTBE_SOURCE_DIGEST="%s"' % digest)
            if verbose:
                print(" ".join(cmd), flush=True)
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
            if verbose and r.stderr.strip():
                print(r.stderr, file=sys.stderr)
        return o

    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    if force or not _newer(LIB, objs):
        cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(force="--incremental" not in sys.argv, verbose=True))
