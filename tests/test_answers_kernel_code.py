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


def test_top_classes_leave_registers_for_eight_wavefronts():
    """64 vector registers to a lane let a SIMD hold eight wavefronts: two workgroups of 1024 threads, four of 512.  Float16 words, which
    cost registers to open, need more with 512 threads, and rows of 16 words a thread fit once."""
    found = {k: v[0] for k, v in mine(registers()).items() if "k_top_long" in k}
    of = lambda threads, words: {("f16" if "IDF16_" in k or "_Float16" in k else "other", v) for k, v in found.items()
                                 if re.search(rf"(Li|, ){threads}(ELi|, ){words}(E|>)", k)}
    for threads, words in ((512, 8), (1024, 4), (1024, 8)):
        some = of(threads, words)
        assert some and all(n <= 64 for kind, n in some if kind == "other" or threads == 1024)
    assert all(n <= 72 for _, n in of(512, 8))                       # seven wavefronts
    assert of(1024, 16) and all(64 < n <= 128 for _, n in of(1024, 16))
