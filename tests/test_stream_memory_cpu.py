"""What the library remembers about streams, on the host: a program may use any number of them, one after the other."""
import subprocess
import sys

from paper_2504_18415_b200 import build, hbl

CODE = """
import ctypes as C, sys
L = C.CDLL(sys.argv[1])
def f(name, result=None):
    g = getattr(L, name)
    g.restype, g.argtypes = result, [C.c_void_p] if result else [C.c_void_p, C.c_bool]
    return g
unflushed, early = f("_ZN3hbl16stream_unflushedEP11CUstream_st", C.c_bool), f("_ZN3hbl21stream_released_earlyEP11CUstream_st", C.c_bool)
set_unflushed, set_early = f("_ZN3hbl20set_stream_unflushedEP11CUstream_stb"), f("_ZN3hbl25set_stream_released_earlyEP11CUstream_stb")
def waiting(s):                        # what a launch of each kind leaves behind
    set_early(s, False)
    set_unflushed(s, True)
def dependent(s, releases=False):
    set_early(s, releases)
    set_unflushed(s, False)
"""


def run(body):
    build.build()
    subprocess.run([sys.executable, "-c", CODE + body, hbl.LIB_PATH], check=True)       # (a process of its own: the memory lasts)


def test_streams_one_after_the_other_leave_nothing_behind():
    run("""
for s in range(1, 2001):
    waiting(s)
    assert unflushed(s) and not early(s)
    dependent(s)
    assert not unflushed(s) and not early(s)
    dependent(s, releases=True)
    assert early(s) and not unflushed(s)
    waiting(s)
    assert unflushed(s) and not early(s)
    dependent(s)
for s in (1, 7, 2001, 5000):
    assert not unflushed(s) and not early(s)
""")


def test_more_streams_at_once_than_there_is_room_for():
    """Those without a place count as out of the ordinary; nothing is taken for ordinary that is not."""
    run("""
for s in range(1, 101):
    waiting(s) if s % 2 else dependent(s, releases=True)
assert all(unflushed(s) for s in range(1, 101, 2)) and all(early(s) for s in range(2, 101, 2))
for s in range(1, 101):
    dependent(s)
for s in range(1, 101):
    waiting(s)
    assert unflushed(s)
    dependent(s, releases=True)
    assert early(s)
""")
