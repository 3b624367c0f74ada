"""Build libgrid.so in-tree for sm_103a with nvcc (host C++ and CUDA sources
compiled in parallel, then linked) and the binding's calls on tensors.  Output:
paper_2607_11951_gb300/_build/libgrid.so and grid_binding.so.  The latter needs
g++ and the headers of Python and torch; where it cannot be built the library is,
with a warning, and all but the model side's calls work."""
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "_build")
SOURCES = ["grid_host.cpp", "grid_kernels.cu", "grid_span.cu", "grid_audit.cu", "grid_kv.cu", "grid_attend.cu",
           "grid_draft.cu", "grid_tree.cu", "grid_pages.cu", "grid_sample.cu"]
NVCC = os.environ.get("NVCC", "nvcc")
FLAGS = ["-gencode", "arch=compute_103a,code=sm_103a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-Xcompiler", "-O2"]


def library_path() -> str:
    return os.path.join(OUT, "libgrid.so")


def binding_path() -> str:
    return os.path.join(OUT, "grid_binding.so")


def build_binding() -> None:
    """The calls on tensors (csrc/grid_python.cpp), against the installed torch; loaded once, so that no symbol is missing."""
    if os.path.exists(binding_path()):
        os.remove(binding_path())  # (none rather than one of other sources)
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("torch is not installed")
    torch = spec.submodule_search_locations[0]
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(NVCC) or "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    libs, tmp = os.path.join(torch, "lib"), binding_path() + ".tmp"
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-shared"] + ["-I" + i for i in include] + \
        [os.path.join(CSRC, "grid_python.cpp"), "-o", tmp, "-L" + libs, "-Wl,-rpath," + libs,
         "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for grid_python.cpp:\n%s%s" % (r.stdout, r.stderr))
    load = "import importlib.machinery as m, importlib.util as u, sys, torch; " \
        "l = m.ExtensionFileLoader('grid_binding', sys.argv[1]); u.module_from_spec(u.spec_from_loader('grid_binding', l))"
    r = subprocess.run([sys.executable, "-c", load, tmp], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("grid_binding.so does not load:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, binding_path())


def build(verbose: bool = False) -> str:
    os.makedirs(OUT, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(OUT, src + ".o")
        cmd = [NVCC] + FLAGS + (["-Xptxas", "-v"] if verbose and src.endswith(".cu") else []) + \
            ["-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s%s" % (src, r.stdout, r.stderr))
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(len(SOURCES) + 1) as ex:
        binding = ex.submit(build_binding)
        objs = list(ex.map(compile_one, SOURCES))
    tmp = library_path() + ".tmp"
    cmd = [NVCC, "-shared", "-gencode", "arch=compute_103a,code=sm_103a"] + objs + ["-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, library_path())
    try:
        binding.result()
    except (RuntimeError, OSError) as e:
        warnings.warn("grid_binding.so was not built, the calls on a model's tensors will not work: %s" % e, RuntimeWarning)
    return library_path()


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
