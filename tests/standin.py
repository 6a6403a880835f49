"""The HIP runtime's part in an operator's call, replaced on the host: a small library, loaded in front of libficco.so in a process of its own, that
notes every launch (kernel, grid, workgroup, LDS) and every LDS limit that is set, by device. So a test sees which kernel a call takes,
and how it launches it, without a GPU; nothing is computed."""
import ctypes as C
import json
import os
import shutil
import subprocess
import sys

import pytest

SOURCE = r"""
#include <cstdio>
#include <map>
#include <string>
#include <vector>
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>
static int g_device = 0, g_cus = 256;
static std::map<const void *, std::string> g_name;
static std::map<std::pair<const void *, int>, int> g_limit;
static std::string g_log;
struct Config { dim3 grid, block; size_t lds; hipStream_t stream; };
static std::vector<Config> g_config;
extern "C" {
void standin_device(int device, int cus) { g_device = device; g_cus = cus; }
// a line a launch: device, kernel, grid, workgroup, LDS of the launch, LDS limit set on that device
const char *standin_log() { return g_log.c_str(); }
void standin_clear() { g_log.clear(); }
const char *standin_kernels()
{
    static std::string all;
    all.clear();
    for (auto &k : g_name) all += k.second + "\n";
    return all.c_str();
}
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *, int *) { g_name[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t s) { g_config.push_back({grid, block, lds, s}); return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s)
{
    *grid = g_config.back().grid; *block = g_config.back().block; *lds = g_config.back().lds; *s = g_config.back().stream;
    g_config.pop_back();
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **, size_t lds, hipStream_t)
{
    char line[512];
    snprintf(line, sizeof line, "%d %s %u %u %u %u %zu %d\n", g_device, g_name[f].c_str(), grid.x, grid.y, grid.z, block.x * block.y * block.z, lds, g_limit[{f, g_device}]);
    g_log += line;
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute, int value) { g_limit[{f, g_device}] = value; return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { *v = g_cus; return hipSuccess; }
hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *, int, size_t lds) { *n = lds > 80 * 1024 ? 1 : 2; return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *at, const void *) { *at = {}; at->type = hipMemoryTypeDevice; at->device = g_device; return hipSuccess; }
}
"""

# what the operators' calls do with the runtime that is replaced here, and nothing else of it
DRIVER = r"""
import ctypes as C, json, sys
sys.path.insert(0, sys.argv[2])
standin = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
import paper_2512_10236_amd as F
standin.standin_log.restype = standin.standin_kernels.restype = C.c_char_p
F.load()
P = 1 << 20
out = []
for c in json.load(sys.stdin):
    device, cus = c.get("device", 0), c.get("cus", 256)
    standin.standin_device(device, cus)
    standin.standin_clear()
    fields, op, given = c["fields"], c["op"], c.get("given", {})
    each = lambda names: [given.get(name, P) for name in names.split()]
    ws = lambda n: given.get("workspace", P if n else None)
    try:
        if op == "linear":
            o = F.ficco_linear_t(**fields)
            n = F.ficco_linear_workspace(o)
            F.ficco_linear(o, *each("A W bias residual pre C"), ws(n), n, None)
        elif op == "linear_backward":
            o = F.ficco_linear_t(**fields)
            n = F.ficco_linear_workspace(o, True)
            F.ficco_linear_backward(o, *each("A W pre dC dA dW dbias"), ws(n), n, None)
        elif op == "norm":
            o = F.ficco_residual_norm_t(**fields)
            n = 0
            F.ficco_residual_norm(o, *each("x block post gate pre y h"), None)
        elif op == "norm_backward":
            o = F.ficco_residual_norm_t(**fields)
            n = F.ficco_residual_norm_workspace(o)
            F.ficco_residual_norm_backward(o, *each("y block post gate pre dy dh dx dblock dpost dgate dpre"), ws(n), n, None)
        elif op == "balance":
            o = F.ficco_expert_balance_t(**fields)
            n = F.ficco_expert_balance_workspace(o)
            F.ficco_expert_balance(o, *each("logits ids valid counts group_valid loss"), ws(n), n, None)
        elif op == "balance_backward":
            o = F.ficco_expert_balance_t(**fields)
            n = 0
            F.ficco_expert_balance_backward(o, *each("logits valid counts group_valid dloss dlogits"), None)
        status = 0
    except F.FiccoError as e:
        status, n = e.status, -1
    out.append(dict(status=status, workspace=n, launches=[l.split() for l in standin.standin_log().decode().splitlines()]))
json.dump(dict(calls=out, kernels=sorted(set(standin.standin_kernels().decode().split()))), sys.stdout)
"""


class Launch:
    def __init__(self, fields):
        self.device, self.kernel = int(fields[0]), fields[1]
        self.grid, self.threads, self.lds, self.limit = tuple(map(int, fields[2:5])), int(fields[5]), int(fields[6]), int(fields[7])


def demangled(names):
    names = list(names)
    r = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True)
    return [n.replace("ficco::", "").replace("(anonymous namespace)::", "").split(">(")[0].replace("void ", "") for n in r.stdout.splitlines()]


def build(folder):
    """The stand-in as a library in `folder`."""
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not shutil.which("c++filt") or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("no compiler for the host, or no HIP headers")
    src, lib = os.path.join(folder, "standin.cpp"), os.path.join(folder, "libstandin.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-I", os.path.join(rocm, "include"), src, "-o", lib], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return lib


def run(lib, calls):
    """(a list of dict(status, workspace, launches) for the calls, all kernels of the library). A call: dict(op, fields of its struct, given: addresses
    of operands in the place of one that is there, device, cus)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", DRIVER, lib, root], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    out = json.loads(r.stdout)
    names = dict(zip(out["kernels"], demangled(out["kernels"])))
    for c in out["calls"]:
        c["launches"] = [Launch(f) for f in c["launches"]]
        for l in c["launches"]:
            l.kernel = names[l.kernel]
    return out["calls"], sorted(names.values())
