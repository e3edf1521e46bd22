"""Static checks over the ISA of the bf16 product kernel (hipcc -S, no GPU): its copies into LDS are inline assembly that the compiler
knows nothing of."""
import re

import pytest

from paper_1804_02941_amd import isa_checks as ic


@pytest.fixture(scope="module")
def product_kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("isa") / "product16.s")
    ic.compile_to_isa("product16.hip", out)
    found = {n: lines for n, lines in ic.kernels(open(out).read()) if "product16_kernel" in n}
    assert len(found) >= 8
    return found


def test_no_copy_reads_a_scalar_register_too_soon(product_kernels):
    for name, lines in product_kernels.items():
        assert any("buffer_load_dwordx4" in l and " lds" in l for l in lines), name
        assert ic.scalar_read_hazards(lines) == [], name


def test_copies_are_waited_for_at_the_barriers_and_nowhere_else_in_the_loop(product_kernels):
    """Every barrier comes with a wait for the wavefront's own copies and reads; and no wait of the compiler's stands among the
    products, where it would hold up the copies that are meant to be in flight."""
    for name, lines in product_kernels.items():
        text = [l.strip() for l in lines]
        for i, l in enumerate(text):
            if l.startswith("s_barrier"):
                assert text[i - 1] == "s_waitcnt vmcnt(0) lgkmcnt(0)", name
        products = [i for i, l in enumerate(text) if l.startswith("v_mfma")]
        waits = [l for l in text[products[0]:products[-1]] if re.match(r"s_waitcnt.*vmcnt", l)]
        assert waits == ["s_waitcnt vmcnt(0) lgkmcnt(0)"], (name, waits)


def test_nothing_else_uses_the_register_of_the_copies_address(product_kernels):
    for name, lines in product_kernels.items():
        users = [l for l in lines if re.search(r"\bm0\b", l.split(";")[0])]
        assert users and all(re.match(r"\s*s_mov_b32 m0, s\d+|\s*s_mov_b32 m0, ttmp", l) for l in users), (name, users[:3])


def test_the_deep_form_leaves_two_steps_of_copies_on_their_way(tmp_path):
    """Four steps in LDS: its barriers wait for all but the copies of two steps (eight each), the first one for all but those of three; and
    no wait of the compiler's for all of them stands among the products."""
    out = str(tmp_path / "product16.s")
    ic.compile_to_isa("product16.hip", out)
    found = [(n, l) for n, l in ic.kernels(open(out).read()) if "product16_deep_kernel" in n]
    assert len(found) == 4
    for name, lines in found:
        assert ic.scalar_read_hazards(lines) == [], name
        text = [l.strip() for l in lines]
        waits = [text[i - 1] for i, l in enumerate(text) if l.startswith("s_barrier")]
        assert waits == [f"s_waitcnt vmcnt({n}) lgkmcnt(0)" for n in (24, 16, 0)], (name, waits)
        products = [i for i, l in enumerate(text) if l.startswith("v_mfma")]
        assert [l for l in text[products[0]:products[-1]] if re.match(r"s_waitcnt.*vmcnt", l)] == ["s_waitcnt vmcnt(16) lgkmcnt(0)"], name


def test_kernels_that_clear_what_lies_behind_a_row(tmp_path):
    """The forms whose words' rows may hold anything behind the width, and the fp32 ones: every barrier comes with the wait for copies and reads
    (what is cleared in LDS included), and among the products of one tile there is no other wait for copies."""
    out = str(tmp_path / "product16.s")
    ic.compile_to_isa("product16.hip", out)
    found = [(n, l) for n, l in ic.kernels(open(out).read()) if "ends_kernel" in n or "product32_kernel" in n]
    assert len(found) == 6 + 8
    for name, lines in found:
        assert ic.scalar_read_hazards(lines) == [], name
        text = [l.strip() for l in lines]
        allowed = (24, 16, 0) if "deep" in name else (0,)
        for i, l in enumerate(text):
            if l.startswith("s_barrier"):
                assert text[i - 1] in [f"s_waitcnt vmcnt({n}) lgkmcnt(0)" for n in allowed], (name, text[i - 1])
        if "ELi256ELi256" in name:                                # (two tiles' code, an end between them)
            continue
        products = [i for i, l in enumerate(text) if l.startswith("v_mfma")]
        for i in range(products[0], products[-1]):
            if re.match(r"s_waitcnt.*vmcnt", text[i]):
                assert text[i + 1].startswith("s_barrier"), (name, text[i])
