"""Build librevnet.so in-tree with nvcc for sm_100a, and _direct.so (the calls from Python that skip ctypes) with g++."""
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librevnet.so")
DIRECT = os.path.join(HERE, "_direct.so")
SOURCES = ["api.cu", "stack.cu", "block.cu", "elementwise.cu", "conv_simt.cu", "conv_tc.cu", "conv_fused.cu", "stem.cu",
           "token_api.cu", "act8.cu", "norm.cu", "wgrad8.cu", "logprobs.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "--use_fast_math=false" if False else "-DREVNET_BUILD"]


def _direct_command():
    """g++ for _direct.so, against the headers of the torch that is installed (None: none is)."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    torch = list(spec.submodule_search_locations)[0]
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", os.path.join(CSRC, "direct.cpp"), "-o", DIRECT,
            "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"],
            "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-L" + HERE, "-l:librevnet.so", "-Wl,-rpath,$ORIGIN"]


def _stale():
    direct = _direct_command() is not None
    if not os.path.exists(LIB) or direct and not os.path.exists(DIRECT):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(DIRECT)) if direct else os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "revnet.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    procs = []
    for s in SOURCES:
        o = os.path.join(objdir, s.replace(".cu", ".o"))
        cmd = ["nvcc", "-c", os.path.join(CSRC, s), "-o", o] + FLAGS + (["-Xptxas", "-v"] if verbose else [])
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    ok = True
    for s, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- {s}\n{out}\n")
        ok = ok and p.returncode == 0
    if not ok:
        raise RuntimeError("nvcc failed")
    objs = [os.path.join(objdir, s.replace(".cu", ".o")) for s in SOURCES]
    subprocess.run(["nvcc", "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a", "-lcudart_static", "-ldl", "-lrt", "-lpthread"],
                   check=True)
    direct = _direct_command()
    if direct:
        subprocess.run(direct, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
