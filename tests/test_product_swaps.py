"""The distances of test_product_waits.py for instructions that write two vector registers: a swap writes its second operand as well as its first."""
import os

import pytest

import test_product_waits as waits
from paper_2602_01410_amd import snip

MFMA = "v_mfma_f32_16x16x32_bf16 a[0:3] v[0:3] v[4:7] a[0:3]".split()


def writes(ins):
    first = first_only(ins)
    return first | waits.registers(ins[2]) if "swap" in ins[0] and ins[0].startswith("v_") else first


first_only = waits.writes


def test_scan_sees_both(monkeypatch):
    swap = "v_permlane16_swap_b32_e32 v9 v4".split()
    assert waits.pairs([swap, MFMA]) == []
    monkeypatch.setattr(waits, "writes", writes)
    assert [w for w, *_ in waits.pairs([swap, MFMA])] == [0] and waits.pairs([swap, "s_nop 1".split(), MFMA]) == []
    assert [w for w, *_ in waits.pairs(["v_swap_b32 v5 v9".split(), "s_nop 0".split(), MFMA])] == [1]


def test_library(monkeypatch, tmp_path):
    if not os.path.exists(waits.OBJDUMP):
        pytest.skip("no disassembler")
    assert os.path.exists(snip.LIB_PATH)
    monkeypatch.setattr(waits, "writes", writes)
    waits.test_library(tmp_path)
