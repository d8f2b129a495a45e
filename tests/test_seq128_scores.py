"""The score products of the 64-rows-per-wave kernels over sequences are inline assembly, as in the
dense kernel: the walk of tests/test_dense128_scores.py over their built instructions finds none
that touches a product's registers too early.  And their copies to LDS take a base from scalar
registers inside inline assembly, where the compiler does not count the 5 wait states behind a
vector instruction that wrote them."""
import os
import re
import subprocess

import pytest

import test_dense128_scores as W


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not (os.path.exists(W.OBJDUMP) and os.path.exists(W.OBJCOPY)):
        pytest.skip("no LLVM binary tools")
    if not os.path.exists(W.LIB):
        pytest.fail("libheadcast.so is not built (run __graft_entry__.build())")
    tmp = tmp_path_factory.mktemp("seq128")
    found = {}
    for n, obj in enumerate(W.device_objects(str(tmp))):
        if b"seq_attn128_kernel" not in obj:
            continue
        path = tmp / f"{n}.o"
        path.write_bytes(obj)
        text = subprocess.run([W.OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        found.update({k: v for k, v in W.kernels(text).items() if "seq_attn128_kernel" in k})
    assert len(found) == 2, sorted(found)
    return found


def test_no_instruction_touches_a_score_too_early(listings):
    for name, code in listings.items():
        products, bad = W.too_early(code)
        assert products >= 64, (name, products)
        assert not bad, (name, bad[:5])


def test_bases_of_copies_are_settled(listings):
    copies = 0
    for name, code in listings.items():
        for i, (_, op, args, _) in enumerate(code):
            m = re.match(r"\s*v\d+, s\[(\d+):(\d+)\]", args)
            if op != "global_load_lds_dwordx4" or not m:
                continue
            copies += 1
            base, waited = set(range(int(m[1]), int(m[2]) + 1)), 0
            for _, before, was, _ in reversed(code[max(0, i - 12):i]):
                if waited >= 5:
                    break
                if before in ("v_readlane_b32", "v_readfirstlane_b32"):
                    w = re.match(r"\s*s(\d+),", was)
                    assert not (w and int(w[1]) in base), (name, i, before, was)
                waited += int(was.strip(), 0) + 1 if before == "s_nop" else 1
    assert copies >= 16
