"""Build librt3d.so (gfx950) in-tree with hipcc.

All HIP code is compiled with packed-fp32 instructions disabled; the host
pass of hipcc warns that it does not know that target feature, which is
harmless.
"""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librt3d.so")
SOURCES = [os.path.join(CSRC, f) for f in (
    "rt3d_host.cpp", "rt3d_kernels.hip", "rt3d_tokens.cpp", "rt3d_norm_rope.hip", "rt3d_attn.hip",
    "rt3d_attn_bwd.hip")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile the library; with force=False an existing build is kept."""
    if not force and os.path.exists(LIB):
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as work:
        objects = [os.path.join(work, os.path.basename(src) + ".o") for src in SOURCES]
        # the sources side by side, then one link
        running = [subprocess.Popen(["hipcc", *FLAGS, "-c", src, "-o", obj], stdout=subprocess.PIPE,
                                    stderr=subprocess.STDOUT, text=True)
                   for src, obj in zip(SOURCES, objects)]
        said = [p.communicate()[0] for p in running]
        failed = [text for p, text in zip(running, said) if p.returncode != 0]
        if failed:
            raise RuntimeError("hipcc failed:\n" + "".join(failed))
        res = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", tmp],
                             capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print("".join(said) + res.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
