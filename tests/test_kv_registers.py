"""The attention kernels over the 4-bit cache keep their sums in ordinary registers.

Beyond 256 registers the compiler moves accumulators to accumulation registers, and was seen to read one
of them back after a loop's last matrix instruction without the wait that it needs (one register of one
tile wrong).  The launch bounds of these kernels prevent that; this reads, in the library as built, what the
compiler reports of every instance."""
import os
import struct
import subprocess

import pytest
import yaml

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2309_01885_amd", "libqe.so")
READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """The gfx950 code objects of the library's bundles."""
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + 1)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    import paper_2309_01885_amd.qe as Q
    Q.load()
    with open(LIB, "rb") as f:
        data = f.read()
    found = {}
    for n, obj in enumerate(code_objects(data)):
        path = tmp_path_factory.mktemp("code") / f"{n}.elf"
        path.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, timeout=60, check=True).stdout
        meta = notes[notes.index("---"):notes.rindex("...")] if "---" in notes else "{}"
        for k in yaml.safe_load(meta).get("amdhsa.kernels", []):
            found[k[".name"]] = k
    return found


def test_no_attention_kernel_uses_accumulation_registers(kernels):
    attn = {n: k for n, k in kernels.items() if "kv_few_kernel" in n or "kv_many_kernel" in n}
    # five widths, three groups (two at 64 channels); few rows: fp32, 16-bit, and two tiles up to 128 channels but in
    # groups of 32 there
    assert len(attn) == 14 * 4 + 7
    for name, k in attn.items():
        assert k[".agpr_count"] == 0, name
        assert k[".vgpr_count"] <= 256, name
