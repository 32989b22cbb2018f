"""The instances of the kernels on 4-bit rows that the library holds are those that some call reaches (no GPU needed)."""
import re
import subprocess

import pytest

from paper_2305_04359_amd import build as B
from test_kernel_resources import READELF

PARTS = {"DF16b": 1, "6__half": 2, "f": 3}  # bf16 numbers for each element of a batch
FEW_BATCH = 96 * 1024                       # bytes of LDS that a batch may take


@pytest.fixture(scope="module")
def instances(tmp_path_factory):
    """{kernel: {(type, numbers...)}}"""
    import struct
    data = open(B.library_path(), "rb").read()
    magic, out = b"__CLANG_OFFLOAD_BUNDLE__", {}
    path = str(tmp_path_factory.mktemp("co") / "code.o")
    for m in re.finditer(magic, data):
        pos = m.start() + len(magic) + 8
        for _ in range(struct.unpack_from("<Q", data, pos - 8)[0]):
            offset, size, idlen = struct.unpack_from("<QQQ", data, pos)
            target = data[pos + 24:pos + 24 + idlen].decode()
            pos += 24 + idlen
            if "gfx950" not in target or size == 0:
                continue
            with open(path, "wb") as f:
                f.write(data[m.start() + offset:m.start() + offset + size])
            notes = subprocess.run([READELF, "--notes", path], capture_output=True, text=True, check=True).stdout
            for name, kind, args in re.findall(r"\.name:\s+_ZN5annmi\d+(mx_\w+?_kernel)I(DF16b|6__half|[fha])?((?:L[ijb]\d+E)*)E", notes):
                out.setdefault(name, set()).add((kind, *(int(x) for x in re.findall(r"L[ijb](\d+)E", args))))
    return out


def test_few_rows(instances):
    """mx_product_few_kernel<T, G, WF, AHEAD, LONG>: 16 (G - 1) + 1 rows and more, of eight steps and more where LONG,
    have to fit in LDS."""
    def fits(kind, g, steps):
        return (16 * g - 15) * (steps * 256 + 16) * PARTS[kind] <= FEW_BATCH

    want = {(kind, g, 2 if g == 1 else 4, 2, 0) for kind in PARTS for g in (1, 2, 3, 4) if fits(kind, g, 1)}
    want |= {(kind, g, 1 if g == 1 else 2, 4 if g == 1 else 2, 1) for kind in PARTS for g in (1, 2, 3, 4) if fits(kind, g, 8)}
    assert instances["mx_product_few_kernel"] == want


def test_many_rows(instances):
    """mx_product_many_kernel<T, XF, WIDE>: up to 64 rows come here if they do not fit in LDS, as those of one step do."""
    want = {(kind, xf, 1) for kind in PARTS for xf in (1, 2)} | {(kind, 2, 0) for kind in PARTS} | {("DF16b", 4, 1)}
    assert instances["mx_product_many_kernel"] == want


def test_quantize(instances):
    """mx_quantize_kernel<T, LPR, WIDE>: rows of fewer than eight elements have one step, which takes 16 lanes."""
    kinds = ("DF16b", "6__half", "f", "h", "a")
    assert instances["mx_quantize_kernel"] == {(kind, lpr, 1) for kind in kinds for lpr in (16, 32, 64)} | {(kind, 16, 0) for kind in kinds}


def test_search(instances):
    """mx_group_many_kernel<STEPS, QF, WR>: eight waves that share 16 QF queries by fours (twos where rows are long) or not."""
    assert instances["mx_group_few_kernel"] == {("", s, q) for s in (1, 2, 3, 4) for q in (1, 2, 4)}
    assert instances["mx_group_many_kernel"] == {("", s, 8, w) for s in (1, 2) for w in (1, 4)} | {("", s, 4, w) for s in (3, 4) for w in (1, 2)}
    assert instances["mx_pick_kernel"] == {("", 256), ("", 1024)}
