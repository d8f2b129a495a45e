"""Built instructions of the kernels with a window: the 64-rows-per-wave kernels' score products are inline assembly, and
the copies to LDS of those and of the gradients take a base from scalar registers inside inline assembly.  The walk of
tests/test_dense128_scores.py finds no instruction that touches a product's registers too early, and none of the copies'
bases are written by a vector instruction within 5 wait states."""
import os
import re
import subprocess

import pytest

import test_dense128_scores as W

KERNELS = {"window_attn128_kernel": 2, "11grad_kernel": 2}


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not (os.path.exists(W.OBJDUMP) and os.path.exists(W.OBJCOPY)):
        pytest.skip("no LLVM binary tools")
    if not os.path.exists(W.LIB):
        pytest.fail("libheadcast.so is not built (run __graft_entry__.build())")
    tmp = tmp_path_factory.mktemp("window")
    found = {}
    for n, obj in enumerate(W.device_objects(str(tmp))):
        if not any(k.encode() in obj for k in KERNELS):
            continue
        path = tmp / f"{n}.o"
        path.write_bytes(obj)
        text = subprocess.run([W.OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        found.update({k: v for k, v in W.kernels(text).items() if any(name in k for name in KERNELS)})
    for name, count in KERNELS.items():
        assert sum(name in k for k in found) == count, (name, sorted(found))
    return found


def test_no_instruction_touches_a_score_too_early(listings):
    for name, code in listings.items():
        if "ILi64E" in name:              # none by hand
            continue
        products, bad = W.too_early(code)
        assert products >= (64 if "window_attn128_kernel" in name else 48), (name, products)
        assert not bad, (name, bad[:5])


def both_halves(text):
    """Vector registers of an operand list, with the accumulation half as 1000 and up."""
    found = W.registers(text)
    for a, b in re.findall(r"(?<![a-z0-9_])a\[(\d+):(\d+)\]", text):
        found.update(range(1000 + int(a), 1001 + int(b)))
    found.update(1000 + int(a) for a in re.findall(r"(?<![a-z0-9_])a(\d+)\b", text))
    return found


def too_late(code):
    """(product, offender): a vector instruction that writes what an inline product reads less than 2 wait states before it.
    (The compiler keeps this distance for products that it knows.)"""
    bad = []
    for i, (_, name, ops, _) in enumerate(code):
        if name != "v_mfma_f32_32x32x16_bf16" or not ops.strip().startswith("v["):
            continue
        reads, waited = both_halves(ops.split(",", 1)[1]), 0
        for _, before, was, target in reversed(code[max(0, i - 4):i]):
            if waited >= 2:
                break
            if before.startswith("v_") and not before.startswith(("v_mfma", "v_cmp", "v_readlane", "v_readfirstlane")):
                if both_halves(was.split(",")[0]) & reads:
                    bad.append((f"{name} {ops.strip()}", f"{before} {was.strip()}"))
                    break
            waited += int(was.strip(), 0) + 1 if before == "s_nop" else 1
    return bad


def test_the_walk_finds_a_late_write():
    mfma = (8, "v_mfma_f32_32x32x16_bf16", " v[0:15], v[32:35], a[0:3], v[0:15]", None)
    for write in (" v34, v7", " a2, v7", " v3, v7"):
        code = [(0, "v_mov_b32_e32", write, None), mfma]
        assert too_late(code)
        assert too_late([code[0], (4, "s_nop", " 0", None), mfma])
        assert not too_late([code[0], (4, "s_nop", " 1", None), mfma])
    assert not too_late([(0, "v_mov_b32_e32", " v36, v34", None), mfma])


def test_products_read_nothing_written_just_before(listings):
    for name, code in listings.items():
        assert "ILi64E" in name or not too_late(code), (name, too_late(code)[:5])


def scalars(args):
    """Scalar registers of the first pair among an instruction's arguments."""
    m = re.search(r"s\[(\d+):(\d+)\]", args)
    return set(range(int(m[1]), int(m[2]) + 1)) if m else set()


def test_bases_of_copies_are_settled(listings):
    for name, code in listings.items():
        copies = 0
        for i, (_, op, args, _) in enumerate(code):
            if op not in ("global_load_lds_dwordx4", "global_load_lds_dword") or not scalars(args):
                continue
            copies += 1
            base, waited = scalars(args), 0
            for _, before, was, _ in reversed(code[max(0, i - 12):i]):
                if waited >= 5:
                    break
                if before.startswith("v_"):
                    # (a vector instruction whose destination is scalar: lane reads, comparisons, carries)
                    first = was.strip().split(",")[0].strip()
                    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", first)
                    wrote = set() if not m else {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))
                    assert not wrote & base, (name, i, before, was)
                waited += int(was.strip(), 0) + 1 if before == "s_nop" else 1
        assert copies >= 4, (name, copies)
