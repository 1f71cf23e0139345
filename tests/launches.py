"""What a call of the library launches, without a device: in a process of its own a few functions of the HIP runtime are replaced
by ones that write launches down.  Pointers are numbers; nothing is dereferenced."""
import ctypes
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAX_ARGS = 16

RECORDER = r"""
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <map>
#include <string>
#include <vector>

struct Dim { uint32_t x, y, z; };
struct Launch { const char *name; Dim grid, block; int64_t args[16]; };
static std::map<const void *, std::string> &names() { static std::map<const void *, std::string> m; return m; }
static std::vector<Launch> &launches() { static std::vector<Launch> v; return v; }
static Dim next_grid, next_block;
static std::string wanted;  // kernels whose first `wanted_args` arguments are kept, 8 bytes each
static int wanted_args = 0;

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *module; return &module; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = device;
}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t, void *) { next_grid = grid, next_block = block; return 0; }
int __hipPopCallConfiguration(Dim *grid, Dim *block, size_t *shared, void **stream)
{
    *grid = next_grid, *block = next_block, *shared = 0, *stream = nullptr;
    return 0;
}
int hipLaunchKernel(const void *f, Dim grid, Dim block, void **args, size_t, void *)
{
    Launch l{names()[f].c_str(), grid, block, {}};
    if (wanted_args && names()[f].find(wanted) != std::string::npos)
        for (int i = 0; i < wanted_args; ++i) std::memcpy(&l.args[i], args[i], sizeof(int64_t));
    launches().push_back(l);
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int *device) { *device = 0; return 0; }
int hipFuncSetAttribute(const void *, int, int) { return 0; }

void recorder_want(const char *name, int args) { wanted = name, wanted_args = args; }
void recorder_clear() { launches().clear(); }
int recorder_count() { return (int)launches().size(); }
const Launch *recorder_at(int i) { return &launches()[i]; }
}
"""


class _Launch(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("grid", ctypes.c_uint32 * 3), ("block", ctypes.c_uint32 * 3),
                ("args", ctypes.c_int64 * MAX_ARGS)]


def build_recorder(folder):
    source, target = os.path.join(folder, "recorder.cpp"), os.path.join(folder, "librecorder.so")
    with open(source, "w") as f:
        f.write(RECORDER)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", source, "-o", target])
    return target


def record(recorder, calls, want="", want_args=0):
    """For each (function, arguments) of `calls` its status and its launches: kernel's name, grid, block and, of kernels with
    `want` in their name, the first `want_args` arguments (as 64 bits; what is narrower lies in the low ones)."""
    job = json.dumps({"recorder": recorder, "calls": calls, "want": want, "args": want_args})
    out = subprocess.run([sys.executable, "-m", "tests.launches"], input=job, cwd=ROOT, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    return json.loads(out.stdout)


def main():
    job = json.load(sys.stdin)
    recorder = ctypes.CDLL(job["recorder"], mode=ctypes.RTLD_GLOBAL)  # (before the library: its symbols come first)
    recorder.recorder_at.restype = ctypes.POINTER(_Launch)
    recorder.recorder_want(job["want"].encode(), job["args"])
    import paper_2511_03586_amd as perf
    results = []
    for name, arguments in job["calls"]:
        recorder.recorder_clear()
        status = getattr(perf, name)(**arguments, check=False)
        launches = [recorder.recorder_at(i).contents for i in range(recorder.recorder_count())]
        results.append({"status": status, "launches": [{"name": l.name.decode(), "grid": list(l.grid), "block": list(l.block),
                                                        "args": list(l.args)[:job["args"]]} for l in launches]})
    json.dump(results, sys.stdout)


if __name__ == "__main__":
    main()
