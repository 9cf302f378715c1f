"""Copies straight into LDS, in the built library's own listing: a vector instruction's scalar result may be read by a memory
instruction five wait states later at the earliest, and the compiler, which keeps that distance elsewhere, does not look into
inline assembly.  So the wait is part of it: s_mov_b32 m0 (one state), s_nop 3 (four), the copy."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2202_00774_amd import binding

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def copies(tmp_path_factory):
    """[(kernel, the two instructions in front, the copy)] of every copy into LDS."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    folder = tmp_path_factory.mktemp("code")
    library = folder / "library.so"
    library.symlink_to(os.path.abspath(binding.library_path()))
    subprocess.run([OBJDUMP, "--offloading", str(library)], cwd=folder, check=True, capture_output=True)

    def listing(path):
        out, name, lines = [], "", []
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)], check=True, capture_output=True, text=True).stdout
        for line in text.splitlines():
            if line.endswith(">:"):
                name, lines = line[line.index("<") + 1:-2], []
            elif line.startswith("\t"):
                line = line.split("//")[0].strip()
                if re.match(r"global_load_lds_|buffer_load_\w+ .*\blds\b", line):
                    out.append((name, lines[-2:], line))
                lines.append(line)
        return out

    objects = sorted(p for p in folder.iterdir() if p.name.endswith("gfx950"))
    assert len(objects) > 50
    with ThreadPoolExecutor(8) as pool:
        return [c for part in pool.map(listing, objects) for c in part]


def late(copies, kind):
    """Those of a kind that read scalar registers, and the ones of them whose own wait is too short."""
    reads = [c for c in copies if c[2].startswith(kind) and re.search(r"\bs(\d|\[)", c[2])]
    own = [re.fullmatch(r"s_mov_b32 m0, \S+ s_nop (\d+)", " ".join(before)) for _, before, _ in reads]
    return reads, sorted({name for (name, _, _), m in zip(reads, own) if m is None or int(m[1]) < 3})


def test_copies_of_tiles_by_buffer_records(copies):
    reads, short = late(copies, "buffer_")
    assert len(reads) > 300 and short == []


def test_copies_from_a_scalar_address(copies):
    reads, short = late(copies, "global_")
    assert len(reads) > 300 and short == []
