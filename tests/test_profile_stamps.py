"""A call whose time is asked for stamps its first launch's begin and its last one's end, however many it makes.  The device runtime's
launch calls are replaced in a client program (tests/profile_client.cpp): no GPU, and no pointer is followed."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
LIB = ROOT / "paper_2206_01299_amd" / "libaqsgd.so"
BEGIN, END = 1, 2


@pytest.fixture(scope="module")
def stamps(tmp_path_factory):
    gxx = shutil.which("g++")
    assert gxx, "g++ is part of the image"
    exe = tmp_path_factory.mktemp("profile") / "client"
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT / 'include'}",
                    str(ROOT / "tests" / "profile_client.cpp"), str(LIB), f"-Wl,-rpath,{LIB.parent}",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", str(exe)], check=True)

    def run(call):
        """The stamps of a call's launches."""
        out = subprocess.run([str(exe), ",".join(str(x) for x in call)], check=True, capture_output=True, text=True).stdout.splitlines()
        assert out[-1] == "call 0"
        return [int(line.split()[1]) for line in out[:-1]]

    return run


@pytest.mark.parametrize("call,launches", [
    (("a", 0, 100, 1), 1), (("a", 0, 100, 64), 1), (("a", 0, 100, 65), 2), (("a", 0, 100, 128), 2), (("a", 0, 100, 200), 4),
    (("a", 2, 1 << 34, 1), 1), (("a", 2, 1 << 34, 2), 2), (("a", 2, 1 << 34, 3), 3), (("a", 2, (1 << 34) - 4096, 2), 1), (("a", 2, 1 << 33, 5), 2),
    (("r", 1, 100, 3), 1), (("r", 1, 10000, 3), 1), (("r", 1, 20000, 3), 2), (("r", 1, 100, 65), 3), (("r", 1, 1 << 34, 200), 5),
    (("g", 1, 10, 1600), 1), (("g", 1, 4096, 1600), 2), (("g", 1, 10, 3), 2), (("g", 1, 10, 70001), 2)])
def test_the_first_launch_stamps_the_begin_and_the_last_one_the_end(stamps, call, launches):
    got = stamps(call)
    assert len(got) == launches
    assert got == ([BEGIN + END] if launches == 1 else [BEGIN, *[0] * (launches - 2), END])
