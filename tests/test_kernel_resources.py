"""What the compiler has allotted to the decode kernels, read from the built library's own metadata.

attend_kernel holds its state in some 230 of 256 vector registers at head_dim 256.  When it had more than that, copies of registers which the
compiler put where a branch of some lanes ends were made for those lanes only, and addresses of the others were lost.  So no kernel
of decoding may need accumulation registers to hold what does not fit, or scratch memory."""
import os
import re
import struct
import subprocess

import pytest

from paper_2403_11805_amd import build

BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """The gfx950 code objects of a library: every bundle is its magic, a count, and that many (offset, size, name)."""
    at = data.find(BUNDLE)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(BUNDLE))
        p = at + len(BUNDLE) + 8
        for _ in range(count):
            off, size, n = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + n].decode()
            p += 24 + n
            if "gfx950" in name and size:
                yield data[at + off:at + off + size]
        at = data.find(BUNDLE, at + len(BUNDLE))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{mangled name: {field of the kernel's metadata: number}}"""
    readelf = os.path.join(os.path.dirname(os.path.realpath(build.hipcc())), "..", "llvm", "bin", "llvm-readelf")
    if not os.path.exists(readelf):
        pytest.skip("needs llvm-readelf beside hipcc")
    with open(build.LIB_PATH, "rb") as f:
        data = f.read()
    found, path = {}, str(tmp_path_factory.mktemp("code") / "object")
    for obj in code_objects(data):
        with open(path, "wb") as f:
            f.write(obj)
        notes = subprocess.run([readelf, "--notes", path], capture_output=True, text=True, check=True).stdout
        for entry in re.split(r"^  - ", notes[notes.index("amdhsa.kernels"):], flags=re.M)[1:]:
            name = re.search(r"^    \.name:\s+'?([\w.]+)", entry, re.M)
            if name:
                found[name.group(1)] = {k: int(v) for k, v in re.findall(r"^(?:    )?\.(\w+):\s+(\d+)$", entry, re.M)}
    return found


@pytest.mark.parametrize("kernel,count", [("append_kernel", 6), ("attend_kernel", 12), ("attend_finish_kernel", 3), ("evict_select_kernel", 5),
                                          ("evict_move_kernel", 3)])
def test_decode_kernels_do_not_spill(kernels, kernel, count):
    mine = {n: k for n, k in kernels.items() if re.search(r"\d%sI" % kernel, n)}
    assert len(mine) == count, sorted(mine)
    for name, k in mine.items():
        spilt = {f: k[f] for f in ("private_segment_fixed_size", "vgpr_spill_count", "agpr_count")}
        assert not any(spilt.values()), (name, spilt)
