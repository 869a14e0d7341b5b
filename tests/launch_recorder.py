"""What the second library would launch, without a GPU: a child process in which hipLaunchKernel is a function that notes the kernel's name, its grid and its
first argument, and launches nothing.  Buffers are addresses that nobody reads."""
import ctypes as C
import json
import os
import re
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#define _GNU_SOURCE
#include <dlfcn.h>
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim;
static void (*note)(const char*, const unsigned*, const unsigned*, void**);
void recorder_note(void (*f)(const char*, const unsigned*, const unsigned*, void**)) { note = f; }
int hipLaunchKernel(const void* kernel, dim grid, dim block, void** args, size_t lds, void* stream) {
  Dl_info at;
  const int known = dladdr(kernel, &at) != 0 && at.dli_sname != NULL;
  if (note) note(known ? at.dli_sname : "?", &grid.x, &block.x, args);
  return 0;
}
"""


class TileArgs(C.Structure):
    """csrc/flux_ffn_tile.h"""
    _fields_ = [("a", C.c_uint64 * 2), ("b", C.c_uint64 * 2), ("sa", C.c_uint64), ("sb", C.c_uint64 * 2)]
    _fields_ += [(n, C.c_uint32) for n in ("pitch_a", "pitch_b", "bytes_a", "bytes_b", "pitch_s")]
    _fields_ += [(n, C.c_int32) for n in ("rows", "cols", "depth", "seg_slabs", "slabs", "full_tiles", "cut_tiles", "parts", "part_slabs", "tiles_m", "tiles_n", "band",
                                          "act", "out_f32", "accumulate", "stream")]
    _fields_ += [("ld", C.c_int64), ("out", C.c_uint64 * 2)] + [(n, C.c_uint64) for n in ("g", "u", "factor", "addend", "partial", "counters")]


class OuterArgs(C.Structure):
    """csrc/flux_loss_few_grad.hip"""
    _fields_ = [("t", TileArgs), ("zt", C.c_uint64), ("xt", C.c_uint64), ("rows_each", C.c_int32)]


WORKSPACE = 99 << 40


def _child():
    """stdin: [shim, [[function, problem's fields, which of its pointers are not null, the workspace's bytes]]]; stdout: status and launches of every call."""
    shim, calls = json.load(sys.stdin)
    shim = C.CDLL(shim, mode=C.RTLD_GLOBAL)                    # (ahead of the runtime: its hipLaunchKernel is the one that is found)
    sys.path.insert(0, ROOT)
    from paper_2406_06858_amd import loss, norm
    launches = []

    @C.CFUNCTYPE(None, C.c_char_p, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32), C.POINTER(C.c_void_p))
    def note(name, grid, block, args):
        name = name.decode()
        seen = {"name": name, "grid": grid[:3], "block": block[:3]}
        cfg = re.search(r"3CfgILi(\d+)ELi(\d+)ELi(\d+)ELi\d+ELi\d+ELi\d+ELb([01])E", name)
        outer = re.search(r"12outer_kernelILi(\d)E", name)
        if outer:
            o = C.cast(args[0], C.POINTER(OuterArgs)).contents
            seen.update(terms=32 * int(outer.group(1)), rows=o.t.rows, cols=o.t.cols, zt=o.zt, xt=o.xt, rows_each=o.rows_each)
        if cfg:
            seen["kind"], seen["bm"], seen["bn"], seen["masked"] = (int(v) for v in cfg.groups())
            t = C.cast(args[0], C.POINTER(TileArgs)).contents
            seen.update({f: list(v) if isinstance(v, C.Array) else v for f, v in ((f, getattr(t, f)) for f, _ in TileArgs._fields_)})
        launches.append(seen)

    shim.recorder_note(note)
    libs, out = {"loss": loss.lib(), "norm": norm.lib()}, []
    for function, fields, pointers, ws in calls:
        launches.clear()
        which = "norm" if "norm" in function else "loss"
        p = (norm.norm_problem if which == "norm" else loss.loss_problem)(**fields)
        # (a terabyte apart)
        args = [(i + 1) << 40 if i in pointers else 0 for i in range(max(pointers) + 1)] + ([] if function == "flux_norm" else [WORKSPACE, ws])
        status = getattr(libs[which], function)(C.byref(p), *args, None)
        out.append({"status": status, "launches": list(launches)})
    json.dump(out, sys.stdout)


def record(tmp_path, calls):
    """[(function, problem's fields, which of its pointers are not null)] -> [{status, launches}].  Pointer i is (i + 1) << 40, the workspace lies at WORKSPACE and is as large as
    any has to be."""
    src, so = tmp_path / "shim.c", tmp_path / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src), "-ldl"], check=True)
    todo = [str(so), [(f, fields, list(pointers), 1 << 50) for f, fields, pointers in calls]]
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], input=json.dumps(todo), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout)


if __name__ == "__main__":
    _child()
