"""Builds libawe.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree, and
the benchmark helper libawe_probe.so (the sustained-MFMA-rate probe).

    python -m paper_2609_24519_amd.build [--resources <out.md>]

``--resources`` also compiles the kernels to assembly and writes the register,
spill and LDS figures the compiler assigned to every kernel (from the code
object metadata).

Every HIP translation unit is compiled with packed FP32 instructions disabled
(-packed-fp32-ops): the kernels' float code must not be turned into
v_pk_*_f32 forms.
"""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libawe.so")
HIP_SOURCES = ["awe_kernels.hip", "awe_small.hip", "awe_rns.hip", "awe_w4.hip", "awe_cache.hip"]
SOURCES = HIP_SOURCES + ["awe_tables.cpp", "awe_api.cpp", "awe_quant_api.cpp"]
PROBE_LIB = os.path.join(HERE, "libawe_probe.so")
PROBE_SOURCES = ["mfma_peak.hip"]
ARCH = "gfx950"


def hipcc():
    for c in (os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc"), "hipcc"):
        if os.path.sep not in c or os.path.exists(c):
            return c
    return "hipcc"


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)


def _compile(sources, lib, verbose):
    """Compiles the sources side by side, four at a time, and links them."""
    with tempfile.TemporaryDirectory() as td:
        objects = [os.path.join(td, s + ".o") for s in sources]
        flags = [hipcc(), "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC",
                 "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                 "-Wall", "-Wno-unused-function", "-I", os.path.join(ROOT, "include")]
        with ThreadPoolExecutor(4) as pool:
            list(pool.map(lambda so: _run(flags + ["-c", os.path.join(CSRC, so[0]), "-o", so[1]], verbose),
                          zip(sources, objects)))
        tmp = lib + ".tmp%d" % os.getpid()
        try:
            _run([hipcc(), "--offload-arch=" + ARCH, "-shared", "-fPIC"] + objects + ["-o", tmp], verbose)
            os.replace(tmp, lib)
        finally:
            if os.path.exists(tmp):
                os.remove(tmp)
    return lib


def build(verbose=False):
    _compile(PROBE_SOURCES, PROBE_LIB, verbose)
    return _compile(SOURCES, LIB, verbose)


def kernel_resources():
    """Per-kernel register / spill / LDS figures from the gfx950 code object metadata: a list of
    (name, vgpr, agpr, sgpr, vgpr spill, sgpr spill, static LDS, scratch, max workgroup) with the
    mangled name's namespace prefix removed."""
    import re

    import yaml

    def metadata(src):
        with tempfile.TemporaryDirectory() as td:
            asm = os.path.join(td, "k.s")
            cmd = [hipcc(), "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC",
                   "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                   "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S",
                   os.path.join(CSRC, src), "-o", asm]
            _run(cmd, False)
            text = open(asm).read()
        return text.split(".amdgpu_metadata", 1)[1].split(".end_amdgpu_metadata", 1)[0].replace("\t", " ")

    rows = []
    with ThreadPoolExecutor(4) as pool:
        for meta in pool.map(metadata, HIP_SOURCES):
            for k in yaml.safe_load(meta)["amdhsa.kernels"]:
                name = re.sub(r"^_ZN3awe12_GLOBAL__N_1", "", k[".name"])
                rows.append((name, k.get(".vgpr_count"), k.get(".agpr_count"), k.get(".sgpr_count"),
                             k.get(".vgpr_spill_count"), k.get(".sgpr_spill_count"),
                             k.get(".group_segment_fixed_size"), k.get(".private_segment_fixed_size"),
                             k.get(".max_flat_workgroup_size")))
    return rows


def resources(out_md):
    """kernel_resources() as a Markdown table."""
    rows = kernel_resources()
    lines = ["# Kernel resources (gfx950 code object metadata)", "",
             "Command: `python -m paper_2609_24519_amd.build --resources %s`" % out_md, "",
             "VGPR is the unified count (arch + accumulation registers); the GEMM's LDS ring is",
             "dynamic (set at launch) and not part of the static LDS column.", "",
             "| kernel (mangled tail) | VGPR | AGPR | SGPR | VGPR spill | SGPR spill | static LDS | scratch | max WG |",
             "|---|---|---|---|---|---|---|---|---|"]
    for r in rows:
        lines.append("| %s | %s | %s | %s | %s | %s | %s | %s | %s |" % r)
    with open(out_md, "w") as f:
        f.write("\n".join(lines) + "\n")


if __name__ == "__main__":
    build(verbose=True)
    if len(sys.argv) == 3 and sys.argv[1] == "--resources":
        resources(sys.argv[2])
    sys.exit(0)
