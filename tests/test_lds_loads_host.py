"""The wait states of loads to LDS that are written as assembly, which the compiler does not look into: read from the gfx950 code that was built."""
import os
import re
import struct
import subprocess

from paper_2510_08318_amd import binding as L

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


def _code_objects(path):
    """The gfx950 images of the bundles in a shared library."""
    data, magic = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        p = at + len(magic) + 8
        for _ in range(struct.unpack_from("<Q", data, p - 8)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24: p + 24 + length].decode()
            p += 24 + length
            if "gfx950" in name and size:
                yield data[at + offset: at + offset + size]
        at = data.find(magic, at + 1)


def _wait_states(ins):
    return int(ins.split()[1], 0) + 1 if ins.startswith("s_nop") else 1


def _written_sgprs(ins):
    """Scalar registers that a vector instruction writes (its first operand)."""
    m = re.match(r"v_\S+\s+s(?:(\d+)\b|\[(\d+):(\d+)\])", ins)
    if not m:
        return set()
    return {int(m.group(1))} if m.group(1) else set(range(int(m.group(2)), int(m.group(3)) + 1))


def test_loads_to_lds_wait_for_their_registers(tmp_path):
    """One wait state from a scalar write of m0 to the load that uses it, five from a vector instruction's write of its scalar address."""
    L.lib()
    loads = 0
    for i, image in enumerate(_code_objects(L.LIB_PATH)):
        path = tmp_path / f"{i}.co"
        path.write_bytes(image)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], check=True, capture_output=True, text=True).stdout
        before, kernel = [], None
        for line in text.splitlines():
            head = re.match(r"[0-9a-f]+ <(.*)>:", line)
            if head:
                before, kernel = [], head.group(1)
                continue
            ins = line.split("//")[0].strip()
            if ins.startswith(("global_load_lds", "buffer_load")) and ("_lds" in ins or ins.endswith("lds")):
                loads += 1
                address = re.search(r"s\[(\d+):(\d+)\]", ins)
                address = set(range(int(address.group(1)), int(address.group(2)) + 1)) if address else set()
                states = 0
                for x in reversed(before):
                    if states >= 5:
                        break
                    assert states >= 1 or not re.match(r"s_\S+\s+m0\b", x), (kernel, x, ins)
                    assert not _written_sgprs(x) & address, (kernel, x, ins)
                    states += _wait_states(x)
            if ins:
                before = (before + [ins])[-6:]
    assert loads > 0
