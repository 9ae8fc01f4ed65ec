"""What the serving operators launch, without a GPU: in a process of its own, where the runtime's calls are a stub's that notes them."""
import json
import subprocess
import sys

import pytest

from conftest import ROOT

STUB = r"""
typedef struct { unsigned x, y, z; } dim;
static int attributes, launches, fail;
static dim grids[16], blocks[16];
static unsigned long lds[16];
int hipFuncSetAttribute(const void *f, int attribute, int value) { (void)f; (void)attribute; (void)value; ++attributes; return fail; }
static dim next_grid, next_block;
static unsigned long next_lds;
int __hipPushCallConfiguration(dim grid, dim block, unsigned long bytes, void *stream)
{
    (void)stream;
    next_grid = grid; next_block = block; next_lds = bytes;
    return 0;
}
int __hipPopCallConfiguration(dim *grid, dim *block, unsigned long *bytes, void **stream)
{
    *grid = next_grid; *block = next_block; *bytes = next_lds; *stream = 0;
    return 0;
}
int hipLaunchKernel(const void *f, dim grid, dim block, void **args, unsigned long bytes, void *stream)
{
    (void)f; (void)args; (void)stream;
    if (launches < 16) { grids[launches] = grid; blocks[launches] = block; lds[launches] = bytes; }
    ++launches;
    return 0;
}
int hipGetLastError(void) { return 0; }
void stub_reset(int error) { attributes = launches = 0; fail = error; }
int stub_attributes(void) { return attributes; }
int stub_launches(void) { return launches; }
unsigned long stub_threads(int i) { return (unsigned long)grids[i].x * blocks[i].x; }
unsigned long stub_lds(int i) { return lds[i]; }
"""

RUN = """
import ctypes as C, json, sys
stub = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
stub.stub_threads.restype = stub.stub_lds.restype = C.c_ulong
sys.path[:0] = [sys.argv[2], sys.argv[2] + "/tests"]
import test_serve_abi as A
from paper_2603_12617_amd import binding as B
L, found = B.lib(), []
for name, cache, over in json.loads(sys.argv[3]):
    seen = []
    for error in (0, 0, 1):                     # twice as it is, once where the attribute cannot be set
        stub.stub_reset(error)
        if name == "sd_pages":
            rc = L.sd_pages(C.byref(A._step(**over)), None)
        elif name == "sd_attend":
            a = A._attention(cache, **over)
            rc = L.sd_attend(C.byref(a), A.ONE, 1 << 50, None)
        else:
            rc = L.sd_verify_logits(C.byref(A._verify(**over)), A.ONE, A.ONE, A.ONE, 1 << 50, None)
        n = stub.stub_launches()
        seen.append([rc, stub.stub_attributes(), [[stub.stub_threads(i), stub.stub_lds(i)] for i in range(n)]])
    found.append(seen)
print("FOUND " + json.dumps(found))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    where = tmp_path_factory.mktemp("stub")
    src, lib = where / "stub.c", where / "stub.so"
    src.write_text(STUB)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", str(lib), str(src)], check=True, timeout=60)

    def run(*calls):
        out = subprocess.run([sys.executable, "-c", RUN, str(lib), ROOT, json.dumps(calls)], capture_output=True, text=True, timeout=120)
        assert out.returncode == 0, out.stderr
        return json.loads([x for x in out.stdout.splitlines() if x.startswith("FOUND ")][0][6:])
    return run


def _heads(D, **over):
    """A cache of 8 heads and a batch of one token each of 64 requests."""
    cache = dict(heads=8, D=D, pages=4096, k_page_stride=128 * D, v_page_stride=128 * D, k_tok_stride=8 * D, v_tok_stride=8 * D, k_head_stride=D, v_head_stride=D)
    batch = dict(B=64, tokens=64, Hq=8, width=64, table_stride=64, q_tok_stride=8 * D, out_tok_stride=8 * D, q_head_stride=D, out_head_stride=D)
    return cache, dict(batch, **over)


def test_shared_memory_beyond_64k_is_asked_for_on_every_call(launches):
    """The attribute is the current device's: a program may have changed that.  Where it cannot be set, nothing is launched."""
    calls = [("sd_attend",) + _heads(128), ("sd_attend",) + _heads(256), ("sd_attend",) + _heads(256, tokens=64 * 40), ("sd_pages", None, dict(B=4096))]
    for call, seen in zip(calls, launches(*calls)):
        for rc, attributes, kernels in seen[:2]:
            assert rc == 0 and attributes == 1 and len(kernels) == 1 and kernels[0][1] > 65536, (call, seen)
        assert seen[2] == [-3, 1, []], (call, seen)
    calls = [("sd_attend",) + _heads(64), ("sd_pages", None, dict(B=64))]
    for call, seen in zip(calls, launches(*calls)):
        assert all(rc == 0 and attributes == 0 and kernels[0][1] <= 65536 for rc, attributes, kernels in seen), (call, seen)


def test_launches_of_more_threads_than_fit_are_refused(launches):
    """A launch has fewer than 2^32 threads a dimension: what needs more is refused, what does not is launched."""
    wide = dict(heads=8192, D=64, page=1, k_page_stride=8192 * 64, v_page_stride=8192 * 64, k_tok_stride=8192 * 64, v_tok_stride=8192 * 64, k_head_stride=64, v_head_stride=64)
    batch = dict(B=2000, tokens=2000, Hq=8192, width=4, table_stride=4, q_tok_stride=8192 * 64, out_tok_stride=8192 * 64)
    rows = dict(B=4000, V=8, p_stride=8, q_stride=8, noise_stride=8)
    calls = [("sd_attend", wide, dict(batch)), ("sd_attend", wide, dict(batch, B=4096, tokens=4096)), ("sd_attend", wide, dict(batch, B=4096, tokens=4096 * 40)),
             ("sd_verify_logits", None, dict(rows, q=None, rows=(1 << 24) - 1)), ("sd_verify_logits", None, dict(rows, q=None, rows=1 << 24)),
             ("sd_verify_logits", None, dict(rows, rows=(1 << 23) + 2000 - 1)), ("sd_verify_logits", None, dict(rows, rows=(1 << 23) + 2000))]
    for (call, (rc, _, kernels)), fits in zip(((c, s[0]) for c, s in zip(calls, launches(*calls))), (True, False, False, True, False, True, False)):
        assert rc == (0 if fits else -2) and bool(kernels) == fits, (call, rc, kernels)
        assert all(0 < threads < 1 << 32 for threads, _ in kernels), (call, kernels)


def test_a_window_beyond_all_keys_is_none(launches):
    """Any window that reaches past the longest context, up to the largest number there is, launches what no window does."""
    one = dict(B=1, tokens=1, width=256, table_stride=256)
    few = dict(B=2, tokens=400, width=256, table_stride=256)
    for batch in (one, few):
        found = [seen[0] for seen in launches(*(("sd_attend", {}, dict(batch, window=w)) for w in (0, 4096, 1 << 40, (1 << 63) - 1, (1 << 63) - 20)))]
        assert all(x == found[0] for x in found) and len(found[0][2]) == 2, found
