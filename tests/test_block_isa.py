"""Static audit of the norms' and the 8-bit calls' machine code (CPU only): no
register spills but in the backward's rows of 1024 threads, where a thread has 128
registers: of fp32, and of bf16 past 8192 columns."""
import re

from test_isa_audit import _compile_to_asm, _functions

SPILL = {("f", 1024, 1), ("f", 1024, 2), ("DF16b", 1024, 2)}  # type, threads and chunks of a row


def test_only_the_widest_rows_spill():
    text = _compile_to_asm("kernels_block.hip")
    found = 0
    for pattern in ("block_norm_fwd_kernel", "block_norm_bwd_kernel", "block_norm_sums_kernel", "act8_pack_kernel",
                    "act8_unpack_kernel"):
        funcs = _functions(text, pattern)
        assert funcs, f"{pattern} not found in the assembly"
        for name, lines in funcs.items():
            of = re.search(r"block_norm_bwd_kernelI(f|DF16b)Li(\d+)ELi(\d+)E", name)
            if of and (of[1], int(of[2]), int(of[3])) in SPILL:
                found += 1
                continue
            assert not [l for l in lines if l.startswith("scratch_")], name
    assert found == len(SPILL)
