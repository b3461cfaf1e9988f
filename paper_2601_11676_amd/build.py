"""Compile the HIP sources under csrc/ into libhalo.so for gfx950 (in-tree).

`python -m paper_2601_11676_amd.build` or `__graft_entry__.build()`.  hipcc
cross-compiles without a GPU present.
"""
import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libhalo.so")

FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fno-fast-math", "-Wall", "-Wextra", "-Wno-unused-parameter",
    # the first kernel arguments arrive in scalar registers with the wave instead of through a load
    # of the argument block: one memory round trip less at the head of every kernel (7B decode step
    # 25.4 -> 24.9 us); kernels keep a prologue that loads them where the dispatcher does not preload
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build(verbose: bool = False, extra=()) -> str:
    extra = list(extra) + os.environ.get("HALO_EXTRA_FLAGS", "").split()
    with tempfile.TemporaryDirectory() as tmp:
        # the files side by side (each is a program of its own to the compiler), then one library of them
        cmds = [["hipcc", *FLAGS, *extra, "-c", "-o", os.path.join(tmp, os.path.basename(s) + ".o"), s] for s in sources()]
        link = ["hipcc", *FLAGS, *extra, "-shared", "-o", OUT, *[c[-2] for c in cmds]]
        if verbose:
            print("\n".join(" ".join(c) for c in (*cmds, link)), flush=True)
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            for done in [pool.submit(subprocess.run, c, check=True) for c in cmds]:
                done.result()
        subprocess.run(link, check=True)
    return OUT


def is_stale() -> bool:
    if not os.path.exists(OUT):
        return True
    t = os.path.getmtime(OUT)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.hpp")) + \
        [os.path.join(os.path.dirname(HERE), "include", "halo.h")]
    return any(os.path.getmtime(p) > t for p in deps)


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
