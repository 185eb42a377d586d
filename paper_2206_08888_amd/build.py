"""Build the HIP library in-tree: python -m paper_2206_08888_amd.build [--trace] [extra hipcc flags]

Every source under csrc/ is compiled for gfx950 with hipcc and linked into
paper_2206_08888_amd/libpop.so.  Packed fp32 VALU ops are switched off for all
device code.  --trace also builds libpop_trace.so, the same library as one
translation unit with the timeline instrumentation compiled in (csrc/trace_unity.hip;
paper_2206_08888_amd/timeline.py uses it).
"""
import os
import re
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

from .spills import partial_stores

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpop.so")
TRACE_LIB = os.path.join(HERE, "libpop_trace.so")
SOURCES = ["pop_api.hip", "k_replay.hip", "k_init.hip", "k_chain.hip", "k_few.hip", "k_act.hip", "k_wgrad_adam.hip", "k_step.hip", "k_sac.hip", "k_wgrad_shared.hip",
           "k_recurrence.hip", "k_linear.hip", "k_clip.hip", "k_orthogonalize.hip", "op_api.hip"]
TRACE_SOURCE = "trace_unity.hip"
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Wno-unused-command-line-argument", "-Wno-pass-failed",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# Vector registers that kernels keep in scratch memory (hipcc has stored one that it spilled right behind an `if` of some lanes for those lanes
# only, and what the others read back was an address).  The operators' kernels (k_recurrence.hip, k_linear.hip, k_clip.hip,
# k_orthogonalize.hip) have none.  These of the engine hold a tile or weights across a product and do not fit: their stores have to be with
# all lanes on, which is looked up in the assembly of every build, the traced one's too (spills.py).
MAY_SPILL = re.compile(r"^_ZN3pop(7k_actor|6k_step|11k_sac_actor)I")


def _hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def _run(cmd):
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in p.stdout.splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if p.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def vector_spills(log):
    """(kernel, vector registers that it spills) for every kernel of hipcc's report on their resources."""
    return [(part.split(None, 1)[0], int(n)) for part in log.split("Function Name: ")[1:] for n in re.findall(r"VGPRs Spill: (\d+)", part)[:1]]


def refuse_spills(source, log, assembly):
    """Raises for kernels that spill vector registers and are not among those that may, or not with all lanes."""
    used = vector_spills(log)
    if len(used) < assembly.count(".amdhsa_kernel "):
        raise RuntimeError("%s: hipcc reports the registers of %d kernels only" % (source, len(used)))
    spilling = [name for name, n in used if n]
    wrong = [name for name in spilling if not MAY_SPILL.match(name)]
    if wrong:
        raise RuntimeError("%s: kernels spill vector registers: %s" % (source, ", ".join(wrong)))
    partial = partial_stores(assembly)
    if partial:
        raise RuntimeError("%s: vector registers are spilled for some lanes only: %s" % (source, "; ".join("%s: %s" % p for p in partial)))


def _compile(cc, source, obj, flags):
    """Compiles one source, looks at what its kernels spill, and returns the compiler's messages."""
    name = os.path.splitext(source)[0]
    work = os.path.join(OBJ, "assembly_" + name)
    shutil.rmtree(work, ignore_errors=True)
    os.makedirs(work)
    try:
        # -save-temps: the object is assembled from the listing that is looked at
        out = _run([cc, *flags, "-Rpass-analysis=kernel-resource-usage", "-save-temps=obj", "-c", os.path.join(CSRC, source), "-o", os.path.join(work, name + ".o")])
        with open(os.path.join(work, name + "-hip-amdgcn-amd-amdhsa-gfx950.s")) as f:
            refuse_spills(source, out, f.read())
        os.replace(os.path.join(work, name + ".o"), obj)
    finally:
        shutil.rmtree(work, ignore_errors=True)
    return "\n".join(l for l in out.splitlines() if "kernel-resource-usage" not in l and "remark" not in l and "|" not in l)


def build(verbose=False, extra_flags=(), trace=False):
    os.makedirs(OBJ, exist_ok=True)
    cc = _hipcc()
    objs = [os.path.join(OBJ, s.replace(".hip", ".o")) for s in SOURCES]

    def one(pair):
        src, obj = pair
        out = _compile(cc, src, obj, [*FLAGS, *extra_flags])
        if src == TRACE_SOURCE:                            # one translation unit, linked by itself
            out += _run([cc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", TRACE_LIB, obj])
        return out

    jobs = ([(TRACE_SOURCE, os.path.join(OBJ, "trace_unity.o"))] if trace else []) + list(zip(SOURCES, objs))      # the long job first
    with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
        logs = list(ex.map(one, jobs))
    logs.append(_run([cc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB, *objs]))
    if verbose:
        print("\n".join(l for l in logs if l.strip()))
    return LIB


if __name__ == "__main__":
    flags = [a for a in sys.argv[1:] if a != "--trace"]
    print(build(verbose=True, extra_flags=flags, trace="--trace" in sys.argv[1:]))
