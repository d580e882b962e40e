"""Builds libxorenc.so (HIP, gfx950) and, where torch is installed, _fp8.so (the calls for torch tensors) in-tree with hipcc.  `python -m paper_1905_10138_amd.build`."""
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
OBJ_DIR = os.path.join(PKG_DIR, "_build")
LIB_PATH = os.path.join(PKG_DIR, "libxorenc.so")
EXT_PATH = os.path.join(PKG_DIR, "_fp8.so")
SOURCES = ["xorenc_host.cpp", "xorenc_paper.cpp", "xorenc_decode.hip", "xorenc_encode.hip", "xorenc_spmm.hip",
           "xorenc_spmm_q1.hip", "xorenc_spmm_q2.hip", "xorenc_spmm_q3.hip", "xorenc_spmm_q4.hip",
           "xorenc_fp8_rows.hip", "xorenc_fp8_matmul.hip", "xorenc_moe.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-munsafe-fp-atomics", "-fvisibility=hidden",
    # packed fp32 VALU forms are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-inline-asm",  # (m0 among the registers that inline assembly changes)
]


def extension_commands(hipcc):
    """Compile and link _fp8.so, against torch's libraries and libxorenc.so beside it."""
    import torch
    base = os.path.dirname(torch.__file__)
    obj = os.path.join(OBJ_DIR, "xorenc_torch_fp8.o")
    compile_it = [hipcc, "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
                  f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-isystem", os.path.join(base, "include"),
                  "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
                  "-isystem", sysconfig.get_paths()["include"],
                  "-isystem", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(hipcc))), "include"), "-Wall",
                  "-c", os.path.join(CSRC, "xorenc_torch_fp8.cpp"), "-o", obj]
    link_it = [hipcc, "-shared", "-fPIC", obj, "-L" + os.path.join(base, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python",
               "-L" + PKG_DIR, "-lxorenc", "-Wl,-rpath,$ORIGIN", "-o", EXT_PATH + ".tmp"]
    return compile_it, link_it


def hipcc_path() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found; libxorenc.so cannot be built")


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + out)
    return out


def build_library(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every source (objects in parallel; HIP for gfx950), link the shared library, and then the extension.  The library
    needs hipcc alone: it is there before an extension that does not build raises, and without torch there is none."""
    hipcc = hipcc_path()
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    cmds = [[hipcc] + FLAGS + ["-x", "hip", "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
    try:
        compile_extension, link_extension = extension_commands(hipcc)
    except ImportError:
        compile_extension = None
        print(f"no torch here: {EXT_PATH} (the calls on 8-bit matrices from Python) is not built")
    with ThreadPoolExecutor(max_workers=max(1, min(jobs, len(cmds) + 1))) as ex:
        extension = ex.submit(_run, compile_extension) if compile_extension else None
        outs = list(ex.map(_run, cmds))
    outs.append(_run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", LIB_PATH + ".tmp"]))
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    if extension:
        outs += [extension.result(), _run(link_extension)]
        os.replace(EXT_PATH + ".tmp", EXT_PATH)
    if verbose:
        for o in outs:
            if o.strip():
                print(o)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
    sys.exit(0)
