"""What the entry points launch, recorded on the CPU: a stand-in for the HIP
runtime's launch call takes down grids and blocks and runs nothing, so that the
largest sizes can be looked at without memory or a GPU, and launches can be
made to fail."""
import ctypes
import json
import subprocess
import sys

import pytest

from paper_2606_03026_amd.build import LIB

SHIM = r"""
#include <stddef.h>
#include <stdint.h>
typedef struct { uint32_t x, y, z; } dim3_t;
static int n, fail_at = -1, error;
static uint64_t grid[64], block[64];
static dim3_t held_grid, held_block;
void shim_reset(int fail) { n = 0; fail_at = fail; error = 0; }
int shim_count(void) { return n; }
uint64_t shim_grid(int i) { return grid[i]; }
uint64_t shim_block(int i) { return block[i]; }
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t shared, void *stream)
{
    (void)shared, (void)stream;
    held_grid = g, held_block = b;
    return 0;
}
int __hipPopCallConfiguration(dim3_t *g, dim3_t *b, size_t *shared, void **stream)
{
    *g = held_grid, *b = held_block, *shared = 0, *stream = NULL;
    return 0;
}
int hipLaunchKernel(const void *f, dim3_t g, dim3_t b, void **args, size_t shared, void *stream)
{
    (void)f, (void)args, (void)shared, (void)stream;
    if (n < 64) {
        grid[n] = (uint64_t)g.x * g.y * g.z;
        block[n] = (uint64_t)b.x * b.y * b.z;
    }
    if (n++ == fail_at)
        error = 9; /* hipErrorInvalidConfiguration */
    return error;
}
int hipGetLastError(void)
{
    const int e = error;
    error = 0;
    return e;
}
"""

CHILD = r"""
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # ahead of the HIP runtime
shim.shim_grid.restype = shim.shim_block.restype = ctypes.c_uint64
lib = ctypes.CDLL(sys.argv[2])
lib.spike_proj_last_error.restype = ctypes.c_char_p
out = []
for name, kinds, args, fail in json.load(sys.stdin):
    f = getattr(lib, name)
    f.argtypes = [{"p": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float}[k] for k in kinds]
    shim.shim_reset(fail)
    rc = f(*args)
    out.append([rc, [[shim.shim_grid(i), shim.shim_block(i)] for i in range(shim.shim_count())]])
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    """record(calls): [(code, [(workgroups, threads of one)])] of (entry point, kinds of its arguments, arguments,
    which of its launches fails or -1)."""
    d = tmp_path_factory.mktemp("shim")
    (d / "shim.c").write_text(SHIM)
    (d / "child.py").write_text(CHILD)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", str(d / "shim.so"), str(d / "shim.c")], check=True)

    def run(calls):
        p = subprocess.run([sys.executable, str(d / "child.py"), str(d / "shim.so"), LIB], input=json.dumps(calls),
                           capture_output=True, text=True, timeout=120)
        assert p.returncode == 0, p.stderr
        return json.loads(p.stdout)

    return run


D = 1 << 40  # addresses that nothing reads
F32, BF16, I64 = 0, 1, 5


def gradient(T, V, dim, grad=BF16, table=BF16, accumulate=0, fail=-1):
    return ["spike_embed_backward", "pilpiiiifipilplp",
            [D, grad, dim, D, I64, T, V, dim, 1.0, accumulate, D, table, dim, D, 1 << 50, None], fail]


def test_zeroing_of_the_largest_tables(record):
    """A launch has fewer than 2^32 threads, whatever the table's rows; with few rows, a workgroup has 8 of them."""
    sizes = [(T, V, dim, table) for T in (0, 1, 24, 25, 100, 2048, 2049, 5000, 1 << 22) for table in (F32, BF16)
             for V, dim in ((1 << 28, 8), (1 << 28, 1), (1 << 28, 64), ((1 << 28) - 3, 9), ((1 << 27) + 1, 16), (1 << 27, 1536),
                            (57344, 1536), (1000003, 256)) if T * dim <= 1 << 35]
    for s, (rc, launches) in zip(sizes, record([gradient(*s[:3], table=s[3]) for s in sizes])):
        assert rc == 0, s
        assert launches and all(g * b < 1 << 32 and g < 1 << 31 for g, b in launches), (s, launches)
    (rc, launches), = record([gradient(0, 57344, 1536)])
    assert launches == [[57344 // 8, 256]]


SPIKE_EHIP = -2


@pytest.mark.parametrize("T,n", [(20, 2), (100, 3), (5000, 4)])
def test_nothing_follows_a_failed_launch_of_the_embedding_gradient(record, T, n):
    """The sums take rows by the keys and positions that the sorting wrote."""
    for fail in range(n):
        (rc, launches), = record([gradient(T, 1000, 64, fail=fail)])
        assert rc == SPIKE_EHIP and len(launches) == fail + 1, (fail, launches)
    (rc, launches), = record([gradient(T, 1000, 64)])
    assert rc == 0 and len(launches) == n


def verify(S, G, V, fail=-1):
    return ["head_draft_verify", "plplipppplpiiippppplp",
            [D, V, D, V, F32, D, None, D, D, V, None, S, G, V, D, D, None, None, D, 1 << 40, None], fail]


def test_nothing_follows_a_failed_launch_of_the_draft_verification(record):
    """The race goes by the statistics and the record that the first kernel wrote or cleared."""
    for S, G, V in ((1, 4, 57344), (64, 4, 57344), (3, 0, 50)):
        for fail, n in ((0, 1), (1, 2)):
            (rc, launches), = record([verify(S, G, V, fail)])
            assert rc == SPIKE_EHIP and len(launches) == n
        (rc, launches), = record([verify(S, G, V)])
        assert rc == 0 and len(launches) == 2


def test_largest_draft_verifications(record):
    sizes = [(S, G, V) for S in (1, 64, 4096) for G in (0, 31) for V in (1, 57344, 1 << 30)]
    for s, (rc, launches) in zip(sizes, record([verify(*s) for s in sizes])):
        assert rc == 0 and all(g * b < 1 << 32 for g, b in launches), (s, launches)
