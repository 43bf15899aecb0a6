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


def versions(torch_version):
    """What _direct.so is built for: the versions of torch and Python whose headers it has inside."""
    return "torch %s, Python %d.%d" % ((torch_version.split("+")[0],) + sys.version_info[:2])


def _torch():
    """-> (folder of the torch that is installed, its version), without importing it (None: none is)."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    folder = list(spec.submodule_search_locations)[0]
    about = {}
    with open(os.path.join(folder, "version.py")) as f:
        for line in f:
            if line.startswith("__version__"):
                exec(line, about)
    return folder, about["__version__"]


def _direct_command():
    """g++ for _direct.so, against the headers of the torch that is installed (None: none is)."""
    found = _torch()
    if found is None:
        return None
    torch, version = found
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", os.path.join(CSRC, "direct.cpp"), "-o", DIRECT, '-DBUILT_FOR="%s"' % versions(version),
            "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(cuda, "include"), "-isystem", sysconfig.get_paths()["include"],
            "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-L" + HERE, "-l:librevnet.so", "-Wl,-rpath,$ORIGIN"]


def _older(target):
    """Whether `target` is missing, or older than one of the sources."""
    if not os.path.exists(target):
        return True
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "revnet.h")]
    return any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _direct_stale():
    found = _torch()
    if found is None:
        return False
    if _older(DIRECT):
        return True
    with open(DIRECT, "rb") as f:                    # the text that the compiler was given stands in it
        return versions(found[1]).encode() + b"\0" not in f.read()


def _build_direct():
    """_direct.so, which the library works without (calls then go through ctypes): where it cannot be built, none is left behind."""
    command = _direct_command()
    if command is None:
        return False
    try:
        r = subprocess.run(command, capture_output=True, text=True)
        why = r.stderr if r.returncode else None
    except OSError as e:
        why = str(e)
    if why is not None:
        if os.path.exists(DIRECT):
            os.remove(DIRECT)
        sys.stderr.write(f"_direct.so is not built; calls on rows of tokens go through ctypes (4 us of host time more each):\n{why}\n")
    return why is None


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _older(LIB):
        if _direct_stale():
            _build_direct()
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
    _build_direct()
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
