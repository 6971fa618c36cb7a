"""The attention's form that the models' decoding takes, queries and outputs as pairs of bf16 planes, against float64.

The C entries offer bf16 and fp32 rows; pairs are reached through the library's own launcher, whose argument structs are
given here field by field and compared with the header's layout before anything is launched."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv as ok
from tests.test_gpu_kv import DEV, Pool, U, attn_bound, bd_, dev, host, starts
from tests.test_gpu_kv_numerics import FORMS

pytestmark = pytest.mark.gpu
I32, I64, VP = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LAUNCH = "_ZN2bd19launch_kv_attentionERKNS_7KvPagesERKNS_10KvAttnArgsEiP12ihipStream_t"
PAIR = 2


class KvPages(ctypes.Structure):
    _fields_ = [("k", VP), ("v", VP), ("ks", VP), ("vs", VP), ("n_pages", I32), ("Hkv", I32), ("hd", I32), ("T", I32)]


class KvRows(ctypes.Structure):
    _fields_ = [("row_start", VP), ("row_cnt", VP), ("pos0", VP), ("table", VP), ("n", I32), ("max_pages", I32), ("rows", I32)]


class KvAttnArgs(ctypes.Structure):
    _fields_ = [("a", KvRows), ("kv_len", VP), ("q", VP), ("out", VP), ("ldq", I64), ("ldo", I64), ("q_plane", I64), ("o_plane", I64),
                ("H", I32), ("B", I32), ("scale_log2", ctypes.c_float), ("inv_B", ctypes.c_double), ("inv_G", ctypes.c_double),
                ("ws", VP), ("ws_bytes", I64), ("max_rows", I32)]


@pytest.fixture(scope="module")
def launch(tmp_path_factory):
    d = tmp_path_factory.mktemp("layout")
    parts = [(s, f) for s in (KvPages, KvRows, KvAttnArgs) for f, _ in s._fields_]
    (d / "l.cpp").write_text('#include "bd_internal.h"\n#include <cstddef>\n#include <cstdio>\nint main() { printf("%d", (int)bd::KVQ_PAIR);\n' +
                             "".join(f'printf(" %zu", sizeof(bd::{s.__name__}));\n' for s in (KvPages, KvRows, KvAttnArgs)) +
                             "".join(f'printf(" %zu", offsetof(bd::{s.__name__}, {f}));\n' for s, f in parts) + "}\n")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([f"{rocm}/bin/amdclang++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include",
                    f"-I{ROOT}/paper_2609_33887_amd/csrc", str(d / "l.cpp"), "-o", str(d / "l")], check=True)
    got = [int(x) for x in subprocess.run([str(d / "l")], check=True, capture_output=True, text=True).stdout.split()]
    want = [PAIR] + [ctypes.sizeof(s) for s in (KvPages, KvRows, KvAttnArgs)] + [getattr(s, f).offset for s, f in parts]
    assert got == want
    f = getattr(bd_().lib, LAUNCH)
    f.argtypes, f.restype = [ctypes.POINTER(KvPages), ctypes.POINTER(KvAttnArgs), ctypes.c_int, VP], ctypes.c_int
    return f


@pytest.mark.parametrize("i", range(len(FORMS)))
@pytest.mark.parametrize("workspace", [True, False])
def test_pairs_against_float64(i, workspace, launch):
    """Every form, keys cut and not, with the models' lengths (keys up to the last row).  Outputs are exact to their two
    planes: 2^-16 of themselves (a plane's rounding, 2^-8, of what the first left, 2^-8) beside the error of fp32
    arithmetic.  The norm: 2^-17 and 4e-6 (as fp32 calls), below 1.2e-5; a lost low plane is 2^-9 of a query or an output."""
    lens, cnt, H, Hkv, hd, T, B, spare = FORMS[i]
    pool = Pool(400 + i, sum(-(-x // T) for x in lens) + 2, Hkv, hd, T)
    table, start, pos0 = pool.tables(lens, spare), starts(cnt), np.array(lens) - cnt
    bd, cache, n, R = bd_(), pool.cache(), len(lens), int(start[-1])
    x = dev(pool.rng.standard_normal((R, H, hd)), torch.float32)
    q = torch.zeros((2, R + 3, H, hd), dtype=torch.bfloat16, device=DEV)           # planes farther apart than the rows
    q[0, :R] = x.bfloat16()
    q[1, :R] = (x - q[0, :R].float()).bfloat16()
    out = torch.full((2, R + 5, H, hd), 9.0, dtype=torch.bfloat16, device=DEV)
    need = bd.bd_kv_attention_workspace(H, Hkv, hd, n, R, max(cnt), T, table.shape[1]) if workspace else 0
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    t, s_, c_, p_ = dev(table), dev(start), dev(cnt), dev(pos0)
    pages = KvPages(cache.k.data_ptr(), cache.v.data_ptr(), cache.k_scale.data_ptr(), cache.v_scale.data_ptr(), cache.n_pages, Hkv, hd, T)
    g = KvAttnArgs(a=KvRows(s_.data_ptr(), c_.data_ptr(), p_.data_ptr(), t.data_ptr(), n, table.shape[1], R), kv_len=None,
                   q=q.data_ptr(), out=out.data_ptr(), ldq=H * hd, ldo=H * hd, q_plane=q.stride(0), o_plane=out.stride(0), H=H, B=B,
                   scale_log2=1.0 / math.sqrt(hd) / math.log(2.0), ws=ws.data_ptr() if need else None, ws_bytes=need, max_rows=max(cnt))
    assert launch(ctypes.byref(pages), ctypes.byref(g), PAIR, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    qs = host(q[0, :R]) + host(q[1, :R])
    ref, mag, big = ok.attention(pool.kc, pool.ks, pool.vc, pool.vs, qs, table, start, pos0, lens, B)
    got = host(out[0, :R]) + host(out[1, :R])
    bound = attn_bound(ref, mag, big, hd, max(lens), torch.float32) + 2.0 ** -16 * np.abs(ref)
    off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    print(f"form {i}: {off:.2e} of the norm")
    assert (np.abs(got - ref) <= bound).all() and off <= 1.2e-5
    assert np.linalg.norm(host(out[0, :R]) - ref) / np.linalg.norm(ref) > 1e-3     # (what the low plane is for)
    assert (host(out[:, R:]) == 9.0).all()
