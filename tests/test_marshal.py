"""The binding's C++ part, on the GPU: what it refuses, and that it lets other threads run."""
import importlib.util
import shutil
import subprocess
import threading
import time

import pytest
import torch

from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from test_parity_attn_q8 import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def test_a_workspace_that_is_not_as_large_as_its_elements():
    """One byte seen as many, and every other byte of a buffer."""
    case = Case([2], [5], 2, 1, 64)
    g = case.dev()
    size = B.adt_tree_attn_q8_workspace_size(**case.shape())
    for ws in (torch.zeros(1, dtype=torch.uint8, device="cuda").expand(size), torch.zeros(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            case.call(g, ws=ws)
    case.call(g)
    case.check(g)


FAKE = """
#include <stdint.h>
#include <time.h>
static int nap(void) { struct timespec t = {0, 400000000}; nanosleep(&t, 0); return 0; }
int adt_norm_rope_qkv(void) { return nap(); }
int adt_kv_compact_q8(void) { return nap(); }
int adt_kv_read_q8(void) { return nap(); }
int adt_tree_attn_q8(void) { return nap(); }
"""


def test_other_threads_run_while_a_call_waits(tmp_path):
    """A launch waits where the device's queue is full: a library in whose place each call sleeps, and a copy of the
    module that calls it."""
    src, so, copy = tmp_path / "fake.c", tmp_path / "fake.so", tmp_path / "_marshal.so"
    src.write_text(FAKE)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    shutil.copy(B.MARSHAL_PATH, copy)
    spec = importlib.util.spec_from_file_location("_marshal", str(copy))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.load(str(so))
    q, pos = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    inv = torch.ones(32, dtype=torch.float64, device="cuda")
    c, s = torch.zeros((1, 1, 1, 4, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros(
        (1, 1, 1, 4), dtype=torch.uint8, device="cuda")
    tree, wide = q.view(1, 2, 1, 64), torch.zeros((1, 1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    calls = [lambda: module.norm_rope_qkv(q, None, None, pos, inv, 1, 1, 64, 0, 1e-6, None, None, None, None, 0, 1.0, q, None, None, None),
             lambda: module.kv_compact_q8(c, c, s, s, pos, None, tree, tree, pos, pos, 1, pos, 1, 1, 64, 1, 4, None),
             lambda: module.kv_read_q8(c, c, s, s, pos, wide, wide, 1, 1, 64, 1, 4, None),
             lambda: module.tree_attn_q8(q.view(2, 1, 64), c[0], c[0], s[0], s[0], pos, tree[0], tree[0], pos, pos, 1, 1, 1, 64, 2, 4, 1.0,
                                         q, None, s.view(-1), None)]
    for call in calls:
        worker = threading.Thread(target=call)
        start = time.perf_counter()
        worker.start()
        time.sleep(0.02)
        assert time.perf_counter() - start < 0.3  # (with the interpreter's lock held, not before the call is over: 0.4)
        worker.join()
        assert time.perf_counter() - start > 0.38
