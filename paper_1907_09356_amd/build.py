"""Compile the HIP library for gfx950 into paper_1907_09356_amd/libchoco.so."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = [os.path.join(HERE, "csrc", name) for name in ("choco.hip", "choco_train.hip", "choco_linear.hip", "choco_linear_f32.hip",
                                                       "choco_linear_bf16.hip", "choco_linear_f16.hip", "choco_muon.hip")]
LIB = os.path.join(HERE, "libchoco.so")

# -ffp-contract=off: every product and sum is rounded on its own, which the
# bit-exact parity of the discrete decisions relies on.  Packed fp32 ops are
# switched off as a precaution against their known mis-roundings.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-ffp-contract=off", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(HERE, "csrc")]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp%d" % os.getpid()
    objects, running = [], []
    try:
        for src in SRC:      # side by side: one of them takes most of the time
            objects.append("%s.%s.o" % (tmp, os.path.basename(src)))
            cmd = ["hipcc"] + FLAGS + ["-c", src, "-o", objects[-1]]
            if verbose:
                print(" ".join(cmd))
            running.append((cmd, subprocess.Popen(cmd)))
        for cmd, p in running:
            if p.wait():
                raise subprocess.CalledProcessError(p.returncode, cmd)
        subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC"] + objects + ["-o", tmp])
        os.replace(tmp, LIB)
    finally:
        for _, p in running:
            p.wait()
        for f in objects:
            if os.path.exists(f):
                os.remove(f)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
