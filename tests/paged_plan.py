"""The plan of paged attention (lpp_paged_plan.h, the header that the calls include), compiled as plain C++ (no GPU): which blocks,
how many ranges of keys, how joined."""
import ctypes as C
import os
import subprocess
from collections import namedtuple

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06352_amd", "csrc")
SOURCE = """
#include "lpp_paged_plan.h"
extern "C" void plan(int32_t bf16, int32_t Hkv, int32_t Dh, int32_t n_cu, int64_t B, int32_t gq, int64_t M, int64_t S, int64_t* out) {
  lpp_paged c;
  c.dtype = bf16 ? LPP_BF16 : LPP_F32; c.Hkv = Hkv; c.Dh = Dh; c.n_cu = n_cu;
  const PagedPlan p = plan_paged(&c, B, gq, M, S);
  const int64_t of[] = {p.shape, p.rows, p.kt, p.wk, p.row_blocks, p.nsplit, p.range, p.join_later, looks_at_lengths(&c, B, p),
                        (int64_t)(p.o_bytes + p.ml_bytes)};
  for (int64_t x : of) *out++ = x;
}
extern "C" int64_t room(int32_t bf16, int32_t Hkv, int32_t Dh, int32_t n_cu, int64_t B, int32_t gq, int64_t M, int64_t S) {
  lpp_paged c;
  c.dtype = bf16 ? LPP_BF16 : LPP_F32; c.Hkv = Hkv; c.Dh = Dh; c.n_cu = n_cu;
  return (int64_t)paged_room(&c, B, gq, M, S);
}
"""
Plan = namedtuple("Plan", "shape rows kt wk row_blocks nsplit range join_later by_lengths bytes")


def build(folder):
    (folder / "t.cpp").write_text(SOURCE)
    inc = ["-I", CSRC, "-I", os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include"), "-I", "/opt/rocm/include"]
    subprocess.run(["g++", "-O1", "-std=c++17", "-ffp-contract=off", "-w", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__"] + inc +
                   [str(folder / "t.cpp"), "-o", str(folder / "t.so")], check=True)
    L = C.CDLL(str(folder / "t.so"))
    L.plan.argtypes, L.plan.restype = [C.c_int32] * 4 + [C.c_int64, C.c_int32, C.c_int64, C.c_int64, C.c_void_p], None

    L.room.argtypes, L.room.restype = [C.c_int32] * 4 + [C.c_int64, C.c_int32, C.c_int64, C.c_int64], C.c_int64

    def plan(dtype, B, H, Hkv, Dh, M, S, n_cu=256):
        out = (C.c_int64 * len(Plan._fields))()
        L.plan(dtype == "bf16", Hkv, Dh, n_cu, B, H // Hkv, M, S, out)
        return Plan(*out)

    def room(dtype, B, H, Hkv, Dh, M, S, n_cu=256):
        return L.room(dtype == "bf16", Hkv, Dh, n_cu, B, H // Hkv, M, S)

    plan.room = room
    return plan
