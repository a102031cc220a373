"""Compile the HIP library for gfx950 in-tree (paper_2511_22481_amd/libomniattn.so), which needs hipcc and nothing else, and the binding's
module that reads torch tensors (paper_2511_22481_amd/gqa_marshal.so, host code), which needs g++ and torch."""
import hashlib
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libomniattn.so")
SOURCES = ["decode_kernels.hip", "decode_mid_kernel.hip", "decode_narrow_kernel.hip", "append_kernels.hip",
           "table_kernels.hip", "gqa_append_kernel.hip", "gqa_decode_kernel.hip",
           "gqa_wide_kernel.hip", "api.cpp", "api_gqa.cpp", "plan.cpp"]
HEADERS = ["kernels.h", "gqa.h", "gqa_common.h", "gqa_deal.h", "plan.h", "decode_common.h", os.path.join("..", "..", "include", "omniattn.h")]

MARSHAL = os.path.join(HERE, "gqa_marshal.so")
MARSHAL_SOURCE = "gqa_marshal.cpp"


def hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


STAMP = LIB + ".stamp"   # hash of the sources the library was built (and checked) from
MARSHAL_STAMP = MARSHAL + ".stamp"
CHECKER = os.path.join(HERE, "check_isa.py")


def source_hash():
    h = hashlib.sha256()
    for f in sorted(SOURCES + HEADERS):
        h.update(f.encode())
        h.update(open(os.path.join(CSRC, f), "rb").read())
    h.update(open(CHECKER, "rb").read())
    return h.hexdigest()


def is_stale():
    """True unless the library exists and was built, and its generated code checked, from
    exactly the present sources (content hash, so that file times do not matter)."""
    if not os.path.exists(LIB) or not os.path.exists(STAMP):
        return True
    return open(STAMP).read().strip() != source_hash()


def build(force=True, verbose=False):
    """hipcc --offload-arch=gfx950, one shared library.  Packed-fp32 code generation
    is switched off for the device pass."""
    if not force and not is_stale():
        return LIB
    if os.path.exists(STAMP):
        os.remove(STAMP)
    cmd = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC", "-shared",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument", "-parallel-jobs=8", "-x", "hip"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES]
    cmd += ["-o", LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
        print("\n".join(l for l in res.stderr.splitlines()
                        if "packed-fp32-ops" not in l))
    if res.returncode != 0:
        raise RuntimeError("hipcc failed")
    check_generated_code(verbose)
    with open(STAMP, "w") as f:     # only a library whose generated code passed the check is stamped
        f.write(source_hash() + "\n")
    return LIB


def marshal_hash():
    """What the module is built from: its sources, one interpreter and one torch."""
    import torch
    h = hashlib.sha256(f"{sys.implementation.cache_tag} {torch.__version__}".encode())
    for f in (MARSHAL_SOURCE, os.path.join("..", "..", "include", "omniattn.h")):
        h.update(open(os.path.join(CSRC, f), "rb").read())
    return h.hexdigest()


def marshal_is_stale():
    """is_stale, of the binding's module."""
    if not os.path.exists(MARSHAL) or not os.path.exists(MARSHAL_STAMP):
        return True
    return open(MARSHAL_STAMP).read().strip() != marshal_hash()


def build_marshal(force=True):
    """The binding's module, with g++ against the torch that is installed."""
    if not force and not marshal_is_stale():
        return MARSHAL
    if os.path.exists(MARSHAL_STAMP):
        os.remove(MARSHAL_STAMP)
    res = subprocess.run(marshal_command(), capture_output=True, text=True)
    if res.returncode != 0:
        print(res.stdout, res.stderr)
        raise RuntimeError("building the binding's module failed")
    with open(MARSHAL_STAMP, "w") as f:
        f.write(marshal_hash() + "\n")
    return MARSHAL


def marshal_command():
    import torch
    root = os.path.dirname(os.path.abspath(torch.__file__))
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(root, "include"), os.path.join(CSRC, MARSHAL_SOURCE),
            "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", MARSHAL]


def check_generated_code(verbose=False):
    """Emit the device assembly of the kernels once more and run the static hazard
    check on it (see check_isa.py); raises if compiler-inserted code reads an MFMA
    result too early."""
    import tempfile
    from .check_isa import check
    problems = []
    with tempfile.TemporaryDirectory() as tmp:
        for src, kernel, builtins in (("decode_kernels.hip", "decode_kernel", False),
                                      ("decode_mid_kernel.hip", "decode_mid_kernel", True),
                                      ("decode_narrow_kernel.hip", "decode_narrow_kernel", False),
                                      ("gqa_decode_kernel.hip", "gqa_decode_kernel", True),
                                      ("gqa_wide_kernel.hip", "gqa_wide_kernel", True)):
            out = os.path.join(tmp, src + ".s")
            cmd = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++20",
                   "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                   "-Wno-unused-command-line-argument", "--cuda-device-only", "-S", "-x", "hip",
                   os.path.join(CSRC, src), "-o", out]
            res = subprocess.run(cmd, capture_output=True, text=True)
            if res.returncode != 0:
                raise RuntimeError("hipcc -S failed:\n" + res.stderr[-2000:])
            problems += check(open(out).read(), kernel, builtins)
    if problems:
        raise RuntimeError("generated code reads MFMA results too early:\n" + "\n".join(problems[:20]))
    if verbose:
        print("ISA hazard check: ok")


if __name__ == "__main__":
    import sys
    sys.path.insert(0, os.path.dirname(HERE))
    from paper_2511_22481_amd.build import build as _b, build_marshal as _m
    print(_b(verbose=True))
    try:
        import torch  # noqa: F401
    except ImportError:
        print("no torch: the binding's module for its tensors is not built")
    else:
        print(_m())
