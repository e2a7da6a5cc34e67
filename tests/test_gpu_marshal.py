"""The argument marshalling module's own behaviour: locks and errors."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STUB = 'extern "C" int refuses(const void*, ...) { throw 1; }\n'
PROGRAM = """
import ctypes, gc, sys, threading
import torch
from paper_2506_07533_b200 import binding as mq
module = mq._native()
real = [ctypes.cast(getattr(mq.lib(), n), ctypes.c_void_p).value for n in
        ("moqae_norm_rope", "moqae_paged_append", "moqae_paged_decode_attn", "moqae_paged_prefill_attn")]
stub = ctypes.cast(ctypes.CDLL(sys.argv[1]).refuses, ctypes.c_void_p).value
q = torch.ones(2, 4, 128, dtype=torch.bfloat16, device="cuda")
pos = torch.arange(2, dtype=torch.int32, device="cuda")
rope = mq.make_rope(mq.rope_table(10, 128), 128)
module.bind(stub, *real[1:])
stop = threading.Event()
other = threading.Thread(target=lambda: [sum(range(1000)) for _ in iter(stop.is_set, True)])
other.start()                      # somebody who takes the interpreter whenever it is free
for _ in range(200):
    try:
        mq.moqae_norm_rope(rope, q, None, pos)
        raise SystemExit("no error")
    except mq.MoqaeError as e:
        assert e.code == mq.ERR_INVALID_ARG
    gc.collect(0)
stop.set()
other.join()
module.bind(*real)
mq.moqae_norm_rope(rope, q, None, pos)
assert torch.equal(q[0], torch.ones_like(q[0]))
print("held")
"""


def test_an_exception_below_the_call_leaves_the_interpreter_locked(tmp_path):
    source, library = tmp_path / "stub.cpp", tmp_path / "stub.so"
    source.write_text(STUB)
    subprocess.check_call(["g++", "-shared", "-fPIC", str(source), "-o", str(library)])
    done = subprocess.run([sys.executable, "-c", PROGRAM, str(library)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.split()[-1] == "held", done.stderr[-2000:]
