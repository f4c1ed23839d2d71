"""Compile the HIP sources under csrc/ for gfx950 into paper_2504_18547_amd/libvitq.so.

hipcc cross-compiles without a GPU.  Flags that matter:
  -ffp-contract=off   every fp32 operation that feeds a quantizer stays a separate, correctly
                      rounded instruction (fma only where the source says fmaf)
  -packed-fp32-ops    disabled: the compiler must not form packed fp32 instructions
"""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libvitq.so")
SOURCES = ["api.hip", "gemm.hip", "attention.hip", "quantize.hip", "layernorm.hip", "gemm_f6.hip", "probe.hip",
           "api_serve.hip", "quantize_e4m3.hip", "gemm_e4m3.hip", "rotate.hip", "attention_paged.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-fno-fast-math", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _headers():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    hs.append(os.path.join(os.path.dirname(HERE), "include", "vitq.h"))
    return hs


def _compile(src, force):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    path = os.path.join(CSRC, src)
    if force or _stale(obj, [path] + _headers()):
        r = subprocess.run([HIPCC] + FLAGS + ["-c", path, "-o", obj], capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
        if err.strip():
            print(err)
    return obj


def build(force: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(lambda s: _compile(s, force), SOURCES))
    if force or _stale(LIB, objs):
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs +
                       ["-Wl,-rpath,/opt/rocm/lib"], check=True)
    return LIB


if __name__ == "__main__":
    print(build())
