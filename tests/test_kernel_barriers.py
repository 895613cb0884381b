"""LDS accesses and barriers of the 8-bit products, from the code built here.

A wave that passes a barrier with reads of LDS in flight may find them
overwritten by another wave's loads to LDS, which start right behind it; nothing
but the distance of memory orders the two.  Every kernel of the 8-bit products
therefore has none in flight at any of its barriers: each path through its
instructions is followed, counting the LDS instructions since the last wait
for them."""
import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
MANY = 64
ENDS = ("s_endpgm", "s_setpc_b64", "s_branch")


def code_objects(lib: str, tmp: str) -> list:
    """The gfx950 code objects of a library, as files."""
    data, out, at = open(lib, "rb").read(), [], 0
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    while (at := data.find(magic, at)) >= 0:
        n, = struct.unpack_from("<Q", data, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(n):
            off, size, idlen = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + idlen].decode()
            p += 24 + idlen
            if "gfx950" in name and size:
                out.append(os.path.join(tmp, f"code{len(out)}.o"))
                with open(out[-1], "wb") as f:
                    f.write(data[at + off:at + off + size])
        at += len(magic)
    return out


def kernels(obj: str) -> dict:
    """{kernel name: [(label, None) or (None, instruction)]}"""
    text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--symbolize-operands", "--no-show-raw-insn", obj],
                          capture_output=True, text=True, check=True).stdout
    found, own = {}, None
    for line in text.splitlines():
        if m := re.match(r"^[0-9a-f]* ?<(.+)>:", line):
            if re.match(r"L\d+$", m.group(1)):
                own.append((m.group(1), None))
            else:
                own = found.setdefault(m.group(1), [])
        elif (m := re.match(r"^\s+([a-z]\S*.*?)\s*(?://.*)?$", line)) and own is not None:
            own.append((None, m.group(1)))
    return found


def most_in_flight(listing: list) -> int:
    """The most LDS instructions that can be in flight at a barrier of a kernel."""
    place = {label: i for i, (label, _) in enumerate(listing) if label}
    seen, todo, worst = {}, [(0, 0)], -1
    while todo:
        i, n = todo.pop()
        while i < len(listing) and seen.get(i, -1) < n:
            seen[i] = n
            label, text = listing[i]
            i += 1
            if label:
                continue
            op = text.split()[0]
            if op.startswith("ds_"):
                n = min(n + 1, MANY)                        # (around a loop that waits for none there is no end)
            elif op == "s_waitcnt" and (m := re.search(r"lgkmcnt\((\d+)\)", text)):
                n = min(n, int(m.group(1)))
            elif op == "s_barrier":
                worst = max(worst, n)
            elif op.startswith(("s_branch", "s_cbranch")):
                todo.append((place[re.search(r"<?(L\d+)>?", text).group(1)], n))
            if op in ENDS:
                break
    return worst


@pytest.fixture(scope="module")
def products(tmp_path_factory):
    lib = os.path.join(ROOT, "paper_2609_35587_amd", "libhwsel.so")
    found = {}
    for obj in code_objects(lib, str(tmp_path_factory.mktemp("code"))):
        if b"k_product_rows" in open(obj, "rb").read():
            found.update({n: v for n, v in kernels(obj).items() if "k_product" in n and not n.endswith(".kd")})
    return found


def test_no_reads_in_flight_at_a_barrier(products):
    most = {name: most_in_flight(listing) for name, listing in products.items()}
    assert sum("k_product_rows" in n for n in most) >= 12 and sum("k_product_deep" in n for n in most) >= 4, sorted(most)
    assert all(n <= 0 for n in most.values()), {k: n for k, n in most.items() if n > 0}
    assert all(most[k] == 0 for k in most if "k_product_join" not in k)      # (each of them has a barrier)


def test_the_count_follows_every_path():
    """Reads before a barrier, behind a branch, around a loop and past a wait that leaves some."""
    def of(*lines):
        return most_in_flight([(t[:-1], None) if t.endswith(":") else (None, t) for t in lines])

    read, wait, barrier = "ds_read_b128 v[0:3], v4", "s_waitcnt lgkmcnt(0)", "s_barrier"
    assert of(read, read, "s_waitcnt vmcnt(8)", barrier, "s_endpgm") == 2
    assert of(read, "s_waitcnt vmcnt(8) lgkmcnt(0)", barrier, "s_endpgm") == 0
    assert of(read, read, read, "s_waitcnt lgkmcnt(1)", barrier, "s_endpgm") == 1
    assert of("L0:", barrier, read, wait, read, "s_cbranch_scc1 L0", "s_endpgm") == 1
    assert of("L0:", read, "s_cbranch_scc1 L0", barrier, "s_endpgm") > 9
    assert of(read, "s_cbranch_scc0 L1", wait, "L1:", barrier, "s_endpgm") == 1
    assert of(read, "s_branch L1", barrier, "L1:", wait, barrier, "s_endpgm") == 0
    assert of(read, "s_endpgm") == -1
