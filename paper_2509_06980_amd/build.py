"""Build librl_rollout.so (HIP, gfx950) in-tree with hipcc, and its binding to torch tensors (host code) with g++."""
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "librl_rollout.so")
TORCH_OUT = os.path.join(HERE, "_policy_torch.so")
COMMON = ["--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-result"]
SOURCES = {
    "kernels_generic.hip": [],
    "kernels_mfma.hip": [],
    # the sampler's integer weights must not see fused multiply-adds
    "kernels_sampler.hip": ["-ffp-contract=off"],
    "kernels_objective.hip": [],
    "kernels_rows.hip": [],
    "kernels_packed_attention.hip": [],
    "kernels_packed_attention_mfma.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_token_logprob.hip": [],
    "kernels_token_logprob_mfma.hip": [],
    "kernels_linear.hip": [],
    "kernels_residual_norm.hip": [],
    "kernels_orthogonal.hip": [],
    "engine.hip": [],
}


def build(verbose=False):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(item):
        src, extra = item
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc, "-c", os.path.join(CSRC, src), "-o", obj] + COMMON + extra
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
        if verbose and r.stderr.strip():
            lines = [l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l]
            if lines:
                print("\n".join(lines), file=sys.stderr)
        return obj

    with ThreadPoolExecutor(4) as ex:
        objs = list(ex.map(compile_one, SOURCES.items()))
    r = subprocess.run([hipcc, "-shared", "--offload-arch=gfx950", "-o", OUT] + objs,
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    build_torch_binding()
    return OUT


def build_torch_binding():
    """_policy_torch.so: the policy update's operators on torch tensors, linked against the library beside it.  None where torch is not
    installed: the engine and the C boundary need none."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    torch = spec.submodule_search_locations[0]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-fPIC", "-shared", "-std=c++17", "-fvisibility=hidden", "-D_GLIBCXX_USE_CXX11_ABI=1",
           "-I" + os.path.join(torch, "include"), "-I" + os.path.join(torch, "include", "torch", "csrc", "api", "include"),
           "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "policy_torch.cpp"), "-o", TORCH_OUT,
           "-L" + os.path.join(torch, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python",
           "-L" + HERE, "-l:librl_rollout.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for policy_torch.cpp:\n{r.stderr}")
    return TORCH_OUT


if __name__ == "__main__":
    print(build(verbose=True))
