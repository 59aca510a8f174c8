"""Other Python threads run while a call of the extension module is inside the library."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# A stand-in for one function of the library, loaded before the package: it takes 0.4 s.
SLOW = """
#include <unistd.h>
int draft_verify(void) { usleep(400000); return 0; }
"""

CALLER = """
import ctypes, sys, threading, time
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
from paper_2501_08090_b200 import binding as b
args = [2, 3, 100, 0, 16, None, 4096, 100, 8192, 100, 64, 96, 128, 256, None]
results = []
thread = threading.Thread(target=lambda: results.append(b._marshal.draft_verify(*args)))
start = time.monotonic()
thread.start()
turns = 0
while thread.is_alive():
    time.sleep(0.002)
    turns += 1
took = time.monotonic() - start
assert results == [0] and took >= 0.4, (results, took)
print(turns)
"""


def test_the_interpreter_is_free_during_a_call(tmp_path):
    from paper_2501_08090_b200 import build
    build.build()
    source, library = tmp_path / "slow.c", tmp_path / "libslow.so"
    source.write_text(SLOW)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(library), str(source)], check=True)
    run = subprocess.run([sys.executable, "-c", CALLER, str(library)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr
    assert int(run.stdout) >= 20                     # about 200 turns of 2 ms; one where the call holds the interpreter
