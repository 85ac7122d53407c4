"""What the compiler made of the kernels of the exchange of answers (built library, no GPU)."""
import re

from kernel_code import instructions, registers


def mine(found):
    return {k: v for k, v in found.items() if "answers" in k}


def test_rows_stay_in_registers():
    """Every kernel keeps its part of a row in vector registers: none are spilled, none of a row's words end in scratch memory."""
    found = mine(registers())
    assert len(found) > 80
    assert not {k: v for k, v in found.items() if v[1]}
    scratch = mine(instructions(lambda body: len(re.findall(r"\bscratch_|\bflat_", body))))
    assert not {k: n for k, n in scratch.items() if n}


def test_two_long_rows_fit_a_compute_unit():
    """512 vector registers to a lane of a SIMD; 512 threads are two wavefronts on each of the four, 1024 are four."""
    found = mine(registers())
    of = lambda kernel, threads: [v[0] for k, v in found.items() if kernel in k and re.search(rf"(Li|, ){threads}(E|,)", k)]
    assert of("k_distill", 512) and max(of("k_distill", 512)) <= 128
    assert of("k_distill", 1024) and max(of("k_distill", 1024)) <= 128


def test_gradients_are_stored_in_16_bytes():
    """at odd addresses too: a store of single elements would be eight of them"""
    stores = mine(instructions(lambda body: len(re.findall(r"global_store_dwordx4", body))))
    of = {k: n for k, n in stores.items() if re.search(r"k_distill.*(Lb1|true)", k)}
    assert len(of) >= 27 and all(of.values())
