"""dig_rope without keys reads the two strides of q and nothing behind them."""
import os
import subprocess
import sys
import textwrap

CODE = """
    import ctypes, mmap
    from paper_2405_18428_b200 import dig
    lib = dig.lib()
    page = mmap.PAGESIZE
    memory = mmap.mmap(-1, 2 * page)
    at = ctypes.addressof(ctypes.c_char.from_buffer(memory))
    libc = ctypes.CDLL(None, use_errno=True)
    assert libc.mprotect(ctypes.c_void_p(at + page), ctypes.c_size_t(page), 0) == 0          # what follows the array cannot be read
    strides = ctypes.c_void_p(at + page - 16)
    ctypes.memmove(strides, (ctypes.c_longlong * 2)(1536, 256), 16)
    one = 0x100000
    status = lib.dig_rope(one, None, strides, one, 1, 1, (ctypes.c_double * 4)(1, 1, 1, 1), (ctypes.c_int * 4)(0, 0, 0, 0), 4, one + (1 << 20), None,
                          2, 6, 4, 0, 64, 0, 0, dig.DIG_BF16, None)
    assert status == dig.DIG_ERR_CUDA, status        # all arguments taken; there is no device to launch on
    libc.mprotect(ctypes.c_void_p(at + page), ctypes.c_size_t(page), 3)
    print("taken")
"""


def test_two_strides_are_enough():
    from paper_2405_18428_b200 import build
    build.build()
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(CODE)], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "taken" in r.stdout, (r.returncode, r.stderr[-500:])
