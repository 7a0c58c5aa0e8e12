"""Builds libnat_hip.so (the C-ABI library) for gfx950 with hipcc, in-tree."""
import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libnat_hip.so")
SOURCES = ["api.hip", "select.hip", "compact.hip", "schedule.hip", "loss_f32.hip", "loss_bf16.hip", "ceilings.hip", "attention.hip",
           "kv_cache.hip", "sample.hip", "heads.hip", "embed.hip", "pages.hip"]
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep packed-fp32 instruction selection off for all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def hipcc():
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def build(verbose=False, extra_flags=(), lib_path=None, obj_dir=None, link_flags=()):
    """Compile every source to an object file (in parallel) and link the shared library.
    lib_path / obj_dir: build somewhere else than in the package (a variant build, e.g. with
    host-side sanitizers); extra_flags go to every compile line, link_flags to the link line."""
    obj_dir = obj_dir or os.path.join(PKG_DIR, "_build")
    lib_path = lib_path or LIB_PATH
    os.makedirs(obj_dir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(obj_dir, src.replace(".hip", ".o"))
        cmd = [hipcc(), *HIPCC_FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    objs = []
    for src, obj, proc in procs:
        out, _ = proc.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if proc.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if verbose and out.strip():
            print(out)
        objs.append(obj)
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *link_flags, *objs, "-o", lib_path]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}")
    return lib_path


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
