"""Builds libdeer_hip.so (the C-ABI HIP library) in-tree for gfx950 with hipcc."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libdeer_hip.so")
SOURCES = ["deer_api.hip", "scan_valu.hip", "scan_gru_fused.hip", "scan_gru_dual.hip", "scan_gru_mh.hip", "gru_newton.hip", "scan_mfma.hip", "chunk_gru.hip", "chunk_gru64.hip", "chunk_gru8.hip", "chunk_cells.hip", "funceval_gru.hip", "cell_lstm.hip", "funceval_mlp.hip", "mlp_vjp.hip", "mlp_general.hip", "mlp_vjp_mfma.hip", "gru_vjp_mfma.hip", "seq_api.hip", "diagrec.hip", "dropout.hip", "matrec.hip", "matrec_grad.hip", "layer_api.hip", "shortconv.hip", "selscan.hip", "selscan_grad.hip", "groupnorm.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# packed fp32 instructions are switched off on purpose: some of their forms have given wrong results on the target machines
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


def _compile(src):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    lines = [ln for ln in r.stdout.splitlines() if "packed-fp32-ops" not in ln]
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, "\n".join(lines)))
    return obj


def build(verbose=False):
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
