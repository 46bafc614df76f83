"""Compiled kernels of the state space scan: distances between matrix-core products, those of
f32 among them, and what reads them.

A bf16 product's result may be read after 8 wait states, one of 16x16x4 f32 values after
10, which is what the compiler leaves before the readers it sees.  Behind a loop it has left
one too few before a store, so the kernels wait eight states of their own there: such a
store lies 8 + 8 - 1 or 10 + 8 - 1 behind the product, along any path of the code.
"""
import os
import shutil
import subprocess

import pytest

import test_mfma_hazards as hazards
from paper_2606_27229_amd import carve

OWN = 8
KINDS = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not os.path.exists(hazards.OBJDUMP):
        pytest.skip("llvm-objdump is not installed")
    carve.load_library()
    at = tmp_path_factory.mktemp("code")
    lib = shutil.copy(carve.LIB_PATH, at / "lib.so")
    subprocess.run([hazards.OBJDUMP, "--offloading", str(lib)], cwd=at, check=True, capture_output=True)
    out = []
    for o in sorted(p for p in os.listdir(at) if p.endswith("gfx950")):
        text = subprocess.run([hazards.OBJDUMP, "-d", "--no-show-raw-insn", str(at / o)], check=True, capture_output=True,
                              text=True).stdout
        # (the scan's functions alone)
        parts = text.split("\n\n")
        text = "\n\n".join(p for p in parts if "carve_ssm_" in p.lstrip("\n").split("\n", 1)[0])
        if any(kind in text for kind in KINDS):
            out.append(text)
    return out


@pytest.mark.parametrize("kind", KINDS)
def test_scan_keeps_its_distances(listings, kind, monkeypatch):
    monkeypatch.setattr(hazards, "PRODUCTS", (kind,))
    monkeypatch.setattr(hazards, "WAIT", KINDS[kind] + OWN - 1)
    assert sum(text.count(kind) for text in listings) > 1000   # (the listings were read)
    bad = []
    for text in listings:
        close = hazards.close_pairs(text)
        if close:
            ops = {fn: {hex(i[0]): i[1] for i in ins} for fn, ins in hazards._listing(text).items()}
            bad += [(fn, ops[fn][b], a, b, d) for fn, a, b, d in close if d < KINDS[kind] or "store" in ops[fn][b]]
    assert not bad, bad[:10]


def test_stores_are_found(monkeypatch):
    """The rule on short listings: the compiler's states alone are too few before a store."""
    product = ("v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], 0", None)
    store, end = ("global_store_dwordx4 v[0:1], v[4:7], off", None), ("s_endpgm", None)
    monkeypatch.setattr(hazards, "WAIT", 8 + OWN - 1)
    assert hazards.close_pairs(hazards._text(product, ("s_nop 7", None), store, end))
    assert not hazards.close_pairs(hazards._text(product, ("s_nop 7", None), ("s_nop 6", None), store, end))
