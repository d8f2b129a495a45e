"""Built instructions of the kernel that gives the logarithms of row sums with waves of 64 rows, by the walks of
tests/test_dense128_scores.py and tests/test_window_code.py: its score products and its copies are those of the other
kernels with a window, placed among other instructions by the compiler."""
import os
import subprocess

import pytest

import test_dense128_scores as W
import test_window_code as C


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not (os.path.exists(W.OBJDUMP) and os.path.exists(W.OBJCOPY)):
        pytest.skip("no LLVM binary tools")
    if not os.path.exists(W.LIB):
        pytest.fail("libheadcast.so is not built (run __graft_entry__.build())")
    tmp = tmp_path_factory.mktemp("logs")
    found = {}
    for n, obj in enumerate(W.device_objects(str(tmp))):
        if b"window_logs128_kernel" not in obj:
            continue
        path = tmp / f"{n}.o"
        path.write_bytes(obj)
        text = subprocess.run([W.OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        found.update({k: v for k, v in W.kernels(text).items() if "window_logs128_kernel" in k})
    assert len(found) == 1
    return found


def test_products_are_apart_from_what_touches_them(listings):
    (name, code), = listings.items()
    products, bad = W.too_early(code)
    assert products >= 64, (name, products)
    assert not bad, (name, bad[:5])
    assert not C.too_late(code), (name, C.too_late(code)[:5])


def test_bases_of_copies_are_settled(listings):
    C.test_bases_of_copies_are_settled(listings)


def test_nothing_is_kept_in_memory(listings):
    (name, code), = listings.items()
    assert not [op for _, op, _, _ in code if op.startswith("scratch_")], name
