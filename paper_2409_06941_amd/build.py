"""Builds libfreeride.so (HIP, gfx950) in-tree with hipcc, and _torch_calls.so, which calls it with torch tensors, with the host's compiler."""
import importlib.util
import os
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfreeride.so")
TORCH_CALLS = os.path.join(HERE, "_torch_calls.so")
SOURCES = ["runtime.cpp", "stage.cpp", "pagerank.hip", "pagerank_prep.hip", "sgd.hip", "gemm.hip", "kv_append.hip", "attend.hip", "sample.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-pthread",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",      # keep packed-fp32 instructions out
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + [os.path.join(CSRC, "common.h"), os.path.join(CSRC, "pr_layout.h"), os.path.join(CSRC, "pr_rules.h"), os.path.join(CSRC, "sgd_rule.h"), os.path.join(CSRC, "gemm_tiles.h"), os.path.join(CSRC, "scratch_pool.h"), os.path.join(CSRC, "lm_types.h"),
                        os.path.join(ROOT, "include", "freeride.h"),
                        os.path.join(ROOT, "include", "freeride_device.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True) -> str:
    """Compile every source into one shared library; returns its path."""
    if not force and not is_stale():
        return LIB
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in sources():                      # one hipcc per source, all at once, then one link
        obj = os.path.join(objdir, os.path.basename(src) + ".o")
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC] + FLAGS + ["-x", "hip", "-c", src, "-o", obj]))
    failed = [p.args for p in procs if p.wait() != 0]
    if failed:
        raise RuntimeError("hipcc failed: %s" % " ".join(failed[0]))
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread"] + objs + ["-o", tmp])
    os.replace(tmp, LIB)
    return LIB


def torch_calls_is_stale() -> bool:
    if not os.path.exists(TORCH_CALLS):
        return True
    t = os.path.getmtime(TORCH_CALLS)
    return any(os.path.getmtime(d) > t for d in (os.path.join(CSRC, "torch_calls.cpp"), os.path.join(ROOT, "include", "freeride.h")))


def build_torch_calls(force: bool = True) -> str:
    if not force and not torch_calls_is_stale():
        return TORCH_CALLS
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    tmp = TORCH_CALLS + ".tmp.%d" % os.getpid()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", os.path.join(ROOT, "include"),
                           "-isystem", os.path.join(torch, "include"), "-isystem", sysconfig.get_paths()["include"],
                           os.path.join(CSRC, "torch_calls.cpp"), "-o", tmp,
                           "-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])
    os.replace(tmp, TORCH_CALLS)
    return TORCH_CALLS


if __name__ == "__main__":
    print(build())
    print(build_torch_calls())
