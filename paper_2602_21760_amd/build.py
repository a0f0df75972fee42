"""Build libhyb.so from csrc/*.hip with hipcc for gfx950 (in-tree, next to this file), and the stand-alone measurement
aids under probes/ (one executable per source, next to it)."""
import concurrent.futures as cf
import glob
import os
import re
import subprocess
import sys

if __package__:
    from . import listing
else:                       # run as a file
    import listing

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libhyb.so")
PROBES = os.path.join(HERE, "probes")

# packed fp32 ops are disabled on purpose (hipcc flag, see the build notes of this target)
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wno-unused-result", "-Wno-unknown-warning-option"]


def _hipcc():
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src):
    obj = os.path.join(OBJ, os.path.basename(src)[:-4] + ".o")
    cmd = [_hipcc()] + HIPCC_FLAGS + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    return obj, r.stderr


def has_asm(src):
    """Inline asm with instructions in it (an empty statement or a wait alone needs no look at the listing)."""
    with open(src) as f:
        return re.search(r'asm[^;]*"[^"]*(ds_read|\bv_)', f.read()) is not None


def listing_of(src):
    """The compiler's listing of a source's kernels, as they are built."""
    cmd = [_hipcc()] + HIPCC_FLAGS + ["--cuda-device-only", "-S", src, "-o", "-"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, r.stderr))
    return r.stdout


def _check_listing(src):
    found = listing.faults(listing_of(src))
    if found:
        raise RuntimeError("the code made from %s is not safe:\n%s" % (src, "\n".join(found)))


def _probe(src):
    exe = src[:-4]
    cmd = [_hipcc()] + [f for f in HIPCC_FLAGS if f != "-fPIC"] + [src, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    return exe, r.stderr


def build(verbose=False, jobs=8):
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    if not srcs:
        raise RuntimeError("no sources under " + CSRC)
    objs = []
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        probes = [ex.submit(_probe, src) for src in sorted(glob.glob(os.path.join(PROBES, "*.hip")))]
        checks = [ex.submit(_check_listing, src) for src in srcs if has_asm(src)]
        for fut in probes:
            _, err = fut.result()
            if verbose and err.strip():
                sys.stderr.write(err)
        for obj, err in ex.map(_compile, srcs):
            objs.append(obj)
            if verbose and err.strip():
                sys.stderr.write(err)
        for fut in checks:
            fut.result()
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
