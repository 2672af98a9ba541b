"""How many threads the scan with matrix states launches: fewer than 2^32 in every launch, or the call is refused before its first one.  Host
only: a stand-in for the runtime's launch, which counts, is loaded before the library."""
import subprocess
import sys

import pytest

import paper_1907_06154_amd as ssam
from test_sequence_abi import DIM, OK

STAND_IN = r"""
int hipGetLastError(void) { return 0; }
int hipGetDevice(int *dev) { *dev = 0; return 0; }
int hipFuncSetAttribute(const void *f, int attr, int value) { (void)f; (void)attr; (void)value; return 0; }
struct dim { unsigned x, y, z; };
int launches;
unsigned long long most;
int __hipPushCallConfiguration(struct dim grid, struct dim block, unsigned long lds, void *stream)
{
    unsigned long long threads = (unsigned long long)grid.x * grid.y * grid.z * block.x * block.y * block.z;
    (void)lds; (void)stream;
    if (threads > most) most = threads;
    return 0;
}
int __hipPopCallConfiguration(struct dim *grid, struct dim *block, unsigned long *lds, void **stream)
{
    *grid = *block = (struct dim){1, 1, 1};
    *lds = 0;
    *stream = 0;
    return 0;
}
int hipLaunchKernel(const void *f, struct dim grid, struct dim block, void **args, unsigned long lds, void *stream)
{
    (void)f; (void)grid; (void)block; (void)args; (void)lds; (void)stream;
    ++launches;
    return 0;
}
"""

PROGRAM = r"""
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
sys.path.insert(0, sys.argv[3])
from test_delta_abi import Delta, DeltaBack, Rows, Seq
name, rest = sys.argv[4], [int(x) for x in sys.argv[5:12]]
dtype, S, H, Hk, K, V, all_ = rest
place = iter(range(1, 99))
at = lambda: next(place) << 46
rows = lambda width: Rows(at(), width, width)          # one row a sequence
common = dict(dtype=dtype, heads=H, key_heads=Hk, key_dim=K, value_dim=V, unit=1, scale=0.1, seq=Seq(S, 1, None, None), q=rows(Hk * K), k=rows(Hk * K),
              v=rows(H * V), g=rows(H), beta=rows(H), q_head=K, k_head=K, v_head=V, work=at(), work_bytes=1 << 58)
if name == "ssam_scan_delta":
    s = Delta(out=rows(H * V), out_head=V, **common)
else:
    s = DeltaBack(grad_out=rows(H * V), grad_out_head=V, marks=at(), grad_v=rows(H * V), **common)
    if all_:
        s.grad_q = rows(Hk * K)
f = getattr(L, name)
f.argtypes = [ctypes.c_char_p, ctypes.c_void_p]
status = f(ctypes.cast(ctypes.byref(s), ctypes.c_char_p), None)
print(status, ctypes.c_int.in_dll(fake, "launches").value, ctypes.c_ulonglong.in_dll(fake, "most").value)
"""
BF16, F32 = 3, 0
FORWARD, BACK = "ssam_scan_delta", "ssam_scan_delta_backward"
# sequences of one row; dtype, sequences, heads, key heads, key, values, whether q's gradient is wanted; launches (0: refused)
CALLS = {"walks of 512 threads": (FORWARD, BF16, 1 << 17, 1, 1, 32, 4096, 0, 0), "one sequence fewer": (FORWARD, BF16, (1 << 17) - 1, 1, 1, 32, 4096, 0, 2),
         "walks of 256 threads": (FORWARD, BF16, 1 << 17, 1, 1, 256, 4096, 0, 2), "fp32": (FORWARD, F32, 1 << 17, 1, 1, 256, 4096, 0, 2),
         "back walks of 512": (BACK, BF16, 1 << 17, 1, 1, 32, 4096, 0, 0), "back, one sequence fewer": (BACK, BF16, (1 << 17) - 1, 1, 1, 32, 4096, 0, 2),
         "rows of 512": (BACK, BF16, 1 << 17, 64, 64, 256, 16, 1, 0), "rows, one sequence fewer": (BACK, BF16, (1 << 17) - 1, 64, 64, 256, 16, 1, 3),
         "rows not wanted": (BACK, BF16, 1 << 17, 64, 64, 256, 16, 0, 2), "fp32 rows of 512": (BACK, F32, 1 << 17, 64, 64, 64, 16, 1, 0)}


@pytest.mark.parametrize("what", CALLS)
def test_no_launch_has_more_threads_than_there_may_be(what, tmp_path):
    name, *numbers, launches = CALLS[what]
    lib = tmp_path / "stand_in.so"
    (tmp_path / "stand_in.c").write_text(STAND_IN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(tmp_path / "stand_in.c")], check=True)
    res = subprocess.run([sys.executable, "-c", PROGRAM, str(lib), ssam.binding.LIB_PATH, __file__.rsplit("/", 1)[0], name, *map(str, numbers)],
                         capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stderr
    status, count, most = map(int, res.stdout.split())
    assert most < 1 << 32, what
    assert (status, count) == ((OK, launches) if launches else (DIM, 0)), (what, res.stdout)
