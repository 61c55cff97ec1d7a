"""The record of streams whose last kernel writes queries, without a device: what the launch of the query transform goes by."""
import os
import subprocess
import sys

from paper_2608_04074_b200 import build

SCRIPT = """
import ctypes, sys, threading
lib = ctypes.CDLL(sys.argv[1])
written, settled, pending = (getattr(lib, f"_Z{len(n)}{n}P11CUstream_st") for n in ("novakv_queries_written", "novakv_queries_settled", "novakv_queries_pending"))
for f in (written, settled, pending):
    f.argtypes, f.restype = [ctypes.c_void_p], None
pending.restype = ctypes.c_bool
LEGACY, PER_THREAD = 1, 2
assert not pending(None) and not pending(64)
written(64); written(64); written(128)
assert pending(64) and pending(128) and not pending(192) and not pending(None)
settled(64)
assert not pending(64) and pending(128)
settled(64); settled(128)
assert not pending(128)
# the default stream has two names; each thread has a stream of its own under one
written(LEGACY)
assert pending(None)
settled(None)
assert not pending(LEGACY)
written(PER_THREAD)
seen = []
t = threading.Thread(target=lambda: (seen.append(pending(PER_THREAD)), settled(PER_THREAD)))
t.start(); t.join()
assert seen == [False] and pending(PER_THREAD)
settled(PER_THREAD)
# more than the record holds: every stream counts as one from then on
for i in range(64):
    written(1024 + 64 * i)
assert not pending(64) and pending(1024)
written(64)
assert pending(64) and pending(192)
settled(64); settled(1024)
assert pending(64) and pending(192)
print("done")
"""


def test_record():
    lib = build.build_cuda()
    # (the handles are no streams: no device may see them)
    run = subprocess.run([sys.executable, "-c", SCRIPT, str(lib)], capture_output=True, text=True, timeout=300,
                         env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert run.returncode == 0 and run.stdout.strip() == "done", run.stderr
