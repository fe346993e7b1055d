"""A CTA that gives up waits for its copies in flight (on the CPU, against a model of mbarriers)."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2311_14114_gb300", "csrc")


def test_giving_up_waits_for_the_copies_in_flight():
    with tempfile.TemporaryDirectory() as tmp:
        exe = os.path.join(tmp, "flights_check")
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "csrc", "flights_check.cpp"),
                        "-o", exe], check=True)
        out = subprocess.run([exe, "20000"], capture_output=True, text=True, check=True, timeout=300).stdout.split()
    early, unnoticed, either, waited, lost_runs = (int(x) for x in out)
    assert early == 0                           # nothing in flight when the waits end well
    assert unnoticed == 0 and lost_runs > 1000
    assert waited > 10000                       # there was something to wait for
    assert either == 0                          # a wait for either parity is over at once, copies in flight or not


def test_the_tile_kernel_uses_it():
    """The kernel that gives up waits through Flights, and asks no barrier for both parities."""
    with open(os.path.join(CSRC, "kv_tile.cu")) as f:
        src = f.read()
    assert "flights.issue(" in src and "flights.land(" in src
    assert not [ln for ln in src.splitlines() if "mbar_try_wait" in ln and ", 0)" in ln and ", 1)" in ln]
