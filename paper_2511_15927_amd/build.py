"""Compile the HIP library for gfx950 into paper_2511_15927_amd/libbimamba.so (in-tree, hipcc), and _calls.so beside it (g++)."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbimamba.so")
CALLS = os.path.join(HERE, "_calls.so")   # the calls around the mixers as functions of torch tensors (host code)
# (d_state, lanes per chain) pairs the scan kernels are instantiated for
VARIANTS = ((4, 1), (8, 1), (16, 1), (16, 2), (16, 4), (32, 1), (32, 2), (32, 4), (64, 1), (64, 4), (128, 1), (128, 4))
# (d_state, head width) pairs of the many-wave chunk walk
SSD_WIDE = ((64, 32), (64, 64), (128, 32), (128, 64))
# packed fp32 VALU forms are switched off for every kernel in this library
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"),
         "-I", CSRC]
NOISE = "is not a recognized feature for this target"


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    log = "\n".join(l for l in r.stdout.splitlines() if NOISE not in l)
    if r.returncode != 0:
        raise RuntimeError("failed: " + " ".join(cmd) + "\n" + log[:4000])
    return log


def sources():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC))] + [os.path.join(ROOT, "include", "bimamba.h")]


def includes_of(src):
    """A source and all that it includes, headers through headers among them."""
    found, todo = set(), [src]
    while todo:
        path = todo.pop()
        if path in found:
            continue
        found.add(path)
        for name in re.findall(r'^#include "([^"]+)"', open(path).read(), re.M):
            todo += [p for p in (os.path.join(CSRC, name), os.path.join(ROOT, "include", name)) if os.path.exists(p)]
    return found


def newest_dep(src):
    """Modification time that an object must beat."""
    return max(os.path.getmtime(p) for p in includes_of(src))


def compile_calls(force):
    """Object of the extension module."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    src, obj = os.path.join(CSRC, "torch_calls.cpp"), os.path.join(OBJ, "torch_calls.o")
    if not force and os.path.exists(obj) and os.path.getmtime(obj) >= newest_dep(src):
        return ""
    includes = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(ROOT, "include")]
    return _run(["g++", "-O2", "-std=c++17", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI] +
                [x for p in includes for x in ("-isystem" if "torch" in p else "-I", p)] + ["-Wall", "-c", src, "-o", obj])


def link_calls():
    """The extension module beside the library, which it finds there; torch's libraries are in the process that imports it."""
    from torch.utils import cpp_extension
    return _run(["g++", "-shared", "-o", CALLS, os.path.join(OBJ, "torch_calls.o"), "-L" + HERE, "-l:libbimamba.so", "-Wl,-rpath,$ORIGIN"] +
                ["-L" + p for p in cpp_extension.library_paths()] + ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])


def build(force: bool = True, jobs: int = 8):
    if not force and os.path.exists(LIB) and os.path.exists(CALLS) and min(map(os.path.getmtime, (LIB, CALLS))) >= max(os.path.getmtime(p) for p in sources()):
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    units = [(os.path.join(CSRC, "bimamba_api.hip"), os.path.join(OBJ, "bimamba_api.o"), [])]
    for n, s in VARIANTS:
        units.append((os.path.join(CSRC, "scan_inst.hip"), os.path.join(OBJ, "scan_n%d_s%d.o" % (n, s)),
                      ["-DBM_N=%d" % n, "-DBM_S=%d" % s]))
    units.append((os.path.join(CSRC, "ssd_inst.hip"), os.path.join(OBJ, "ssd_inst.o"), []))
    units.append((os.path.join(CSRC, "ssd_block_inst.hip"), os.path.join(OBJ, "ssd_block_inst.o"), []))
    for n, p in SSD_WIDE:
        units.append((os.path.join(CSRC, "ssd_wide_inst.hip"), os.path.join(OBJ, "ssd_wide_n%d_p%d.o" % (n, p)),
                      ["-DBM_N=%d" % n, "-DBM_P=%d" % p]))
    units.append((os.path.join(CSRC, "bwd_inst.hip"), os.path.join(OBJ, "bwd_inst.o"), []))
    units.append((os.path.join(CSRC, "row_inst.hip"), os.path.join(OBJ, "row_inst.o"), []))
    units.append((os.path.join(CSRC, "stack_inst.hip"), os.path.join(OBJ, "stack_inst.o"), []))
    for name in ("embed", "norm", "scores", "clip"):
        units.append((os.path.join(CSRC, name + ".hip"), os.path.join(OBJ, name + ".o"), []))
    todo = [u for u in units if force or not os.path.exists(u[1]) or os.path.getmtime(u[1]) < newest_dep(u[0])]
    cmds = [["hipcc"] + FLAGS + extra + ["-c", src, "-o", obj] for src, obj, extra in todo]
    with ThreadPoolExecutor(max_workers=max(1, min(jobs, len(cmds) + 1))) as ex:
        calls = ex.submit(compile_calls, force)
        logs = list(ex.map(_run, cmds))
    logs.append(_run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [u[1] for u in units]))
    logs.append(calls.result())   # (the library is there by now: it needs neither g++ nor the headers of Python and torch)
    logs.append(link_calls())
    out = "\n".join(l for l in logs if l.strip())
    if out.strip():
        print(out)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--incremental" not in sys.argv))
