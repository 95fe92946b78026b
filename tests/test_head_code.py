"""The machine code of the head's kernels, as the build made it from this repository's sources: waits that the hardware leaves to the program and
that the compiler does not put into inline assembly."""
import os
import re
import subprocess

import pytest

from paper_2411_18462_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    """Instructions of the library's gfx950 code, (name, operands), in the order of their addresses."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    here = tmp_path_factory.mktemp("code")
    os.symlink(build.LIB, here / "libsvip.so")                     # (the parts of the library are written beside it)
    subprocess.run([OBJDUMP, "--offloading", "libsvip.so"], cwd=here, check=True, stdout=subprocess.DEVNULL)
    parts = sorted(f for f in os.listdir(here) if "gfx950" in f)
    assert len(parts) == len(build.SOURCES)
    out = []
    for part in parts:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], cwd=here, check=True, stdout=subprocess.PIPE, text=True).stdout
        out += re.findall(r"^\t(\S+)[ \t]*(.*?)[ \t]*//", text, re.M)
    return out


def before(listing, i, states):
    """Instructions that come fewer than that many wait states ahead of instruction i."""
    for name, args in reversed(listing[max(0, i - states):i]):
        if states <= 0:
            return
        yield name, args
        states -= int(args.split()[0], 0) + 1 if name == "s_nop" else 1


def scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    return set() if not m else {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def test_copies_into_lds_wait_for_what_they_read(listing):
    """One wait state between a write of M0 and the copy that takes its LDS address from it; five between a vector instruction's write of a scalar
    register and a copy whose base it is."""
    copies = 0
    for i, (name, args) in enumerate(listing):
        if not name.startswith("global_load_lds"):
            continue
        copies += 1
        assert not any(re.match(r"m0\b", a) for _, a in before(listing, i, 1)), listing[i - 3:i + 1]
        base = scalars(args.split(", ")[1])
        for n, a in before(listing, i, 5):
            if n.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
                assert not scalars(a) & base, listing[i - 6:i + 1]
    assert copies > 1000                                             # (all of a library's tiles: the listing was understood)
