"""Builds libsamkv.so (sm_100a only) in-tree with nvcc, and the binding's extension module with g++.  `python -m paper_2508_11661_b200.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import warnings

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libsamkv.so")
DEBUG_LIB_PATH = os.path.join(PKG_DIR, "libsamkv_debug.so")   # same sources with -DSAMKV_DEBUG_CHECKS (test hooks)
MARSHAL_PATH = os.path.join(PKG_DIR, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))   # (names the interpreter it is for)
SOURCES = ["api.cu", "score.cu", "score_static.cu", "select.cu", "topp.cu", "align.cu", "means.cu", "compact.cu", "attn.cu", "attn_mma.cu", "attn_tc2.cu", "attn_tc3.cu", "attn_tc4.cu",
           "packed_api.cu", "packed_append.cu", "packed_pages.cu", "packed_scores.cu", "packed_attn.cu", "packed_tc.cu", "packed_tc_mask.cu", "packed_tc_cap.cu", "packed_tc_bias.cu", "packed_score_plan.cu", "packed_decode.cu", "packed_decode_scores.cu", "packed_f32.cu", "packed_f32_scores.cu"]


def nvcc_path() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def build_marshal(force: bool = False) -> str:
    """The binding's argument checks (csrc/marshal.cpp) as an extension module next to it, for this interpreter and this torch
    (a file beside it says for which; the binding looks, too)."""
    import torch
    src = os.path.join(CSRC, "marshal.cpp")
    newest = max(os.path.getmtime(f) for f in (src, os.path.join(ROOT, "include", "samkv.h")))
    made_for = MARSHAL_PATH + ".torch"
    if not force and os.path.exists(MARSHAL_PATH) and os.path.exists(made_for) and os.path.getmtime(MARSHAL_PATH) >= newest:
        with open(made_for) as f:
            if f.read() == torch.__version__:
                return MARSHAL_PATH
    for old in (MARSHAL_PATH, made_for):                 # one that does not fit must not stay where a build fails
        if os.path.exists(old):
            os.remove(old)
    t, part = os.path.dirname(torch.__file__), f"{MARSHAL_PATH}.{os.getpid()}"
    try:
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC",
                               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                               f'-DSAMKV_TORCH_VERSION="{torch.__version__}"',
                               "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
                               "-I", os.path.join(t, "include"), "-I", os.path.join(t, "include", "torch", "csrc", "api", "include"),
                               src, "-o", part, "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
                               f"-Wl,-rpath,{os.path.join(t, 'lib')}"])
        os.replace(part, MARSHAL_PATH)
    finally:
        if os.path.exists(part):
            os.remove(part)
    with open(made_for, "w") as f:
        f.write(torch.__version__)
    return MARSHAL_PATH


def _optional_marshal(force: bool) -> None:
    """The library needs no extension module, and the binding does with its Python forms where there is none."""
    try:
        build_marshal(force)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"the binding's extension module (_marshal) was not built, its Python forms are used: {e}", RuntimeWarning)


def _stale(lib_path: str = LIB_PATH) -> bool:
    if not os.path.exists(lib_path):
        return True
    t = os.path.getmtime(lib_path)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != "marshal.cpp"] + [os.path.join(ROOT, "include", "samkv.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """debug=True builds libsamkv_debug.so: the same library plus the hooks a test needs to make a bounded wait run out."""
    lib_path = DEBUG_LIB_PATH if debug else LIB_PATH
    _optional_marshal(force)
    if not force and not _stale(lib_path):
        return lib_path
    objs = []
    build_dir = os.path.join(PKG_DIR, "build", "debug" if debug else "release")
    os.makedirs(build_dir, exist_ok=True)
    common = [nvcc_path(), "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if debug:
        common += ["-DSAMKV_DEBUG_CHECKS"]
    if verbose:
        common += ["-Xptxas", "-v"]
    procs = []
    for src in SOURCES:
        obj = os.path.join(build_dir, src.replace(".cu", ".o"))
        objs.append(obj)
        procs.append((src, subprocess.Popen(common + ["-c", os.path.join(CSRC, src), "-o", obj],
                                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    subprocess.check_call([nvcc_path(), "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", lib_path] + objs)
    return lib_path


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv, debug=True))
