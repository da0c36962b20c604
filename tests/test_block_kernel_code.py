"""What the compiler made of the drafting step on a 4-bit cache, read from the library's own code object: properties that its speed
rests on and no result shows."""
import re

from test_kernel_code import _tile_loops, _tool, code_objects  # noqa: F401  (a fixture)

KERNEL = re.compile(r"draft_scaled_kernelILi(\d+)ELNS_9CacheTypeE2ELi(\d)ELi(\d)ELi(\d)ELb(\d)E")


def test_loops_wait_for_no_load_of_unknown_memory(code_objects):  # noqa: F811
    """A load that might be from LDS (flat) counts with the LDS accesses: the loops would wait for memory with every tile.  Widened
    values stand in vector registers: nothing in the loops is reloaded from scratch memory or, as a parameter, from memory."""
    seen = set()
    for co in code_objects:
        for kernel, body in _tile_loops(_tool("llvm-objdump", "-d", "--no-show-raw-insn", co)):
            m = KERNEL.search(kernel)
            if m and any("pk_bf16_fp4" in x for x in body):
                seen.add(m.groups())
                assert not [x for x in body if x.startswith(("flat_", "scratch_", "s_load"))], kernel
    # D, row blocks, waves of a stream, waves, long runs: those whose loop holds 16 matrix instructions or more
    assert {("64", "2", "1", "4", "0"), ("64", "2", "2", "4", "0"), ("128", "1", "1", "8", "0"), ("128", "1", "2", "4", "0"), ("128", "1", "4", "8", "0")} <= seen, seen


def test_the_workgroups_that_the_launch_means_fit_a_cu(code_objects):  # noqa: F811
    """Two workgroups of four waves, or one of eight, a CU; at D = 64 with one block of rows two of eight."""
    seen = set()
    for co in code_objects:
        for lds, name, vgprs in re.findall(r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+(\S+).*?\.vgpr_count:\s+(\d+)",
                                           _tool("llvm-readobj", "--notes", co), re.S):
            m = KERNEL.search(name)
            if m:
                D, rows, parts, waves, long_runs = (int(x) for x in m.groups())
                n = 2 if waves == 4 or (D == 64 and rows == 1 and not long_runs) else 1
                seen.add(m.groups())
                assert int(lds) * n <= 160 * 1024 and int(vgprs) * n * waves // 4 <= 512, (name, lds, vgprs)
    assert len(seen) == 11, seen
