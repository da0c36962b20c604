"""What the compiler made of the kernels that move rows to and from a cache, read from the library's own code object."""
import re

from test_kernel_code import _tool, code_objects  # noqa: F401  (a fixture)


def _kernels(code_objects, name):  # noqa: F811
    """(name, instructions) of every form of a kernel."""
    for co in code_objects:
        kernel, body = "", []
        for line in _tool("llvm-objdump", "-d", "--no-show-raw-insn", co).splitlines() + ["0 <end>:"]:
            label = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
            if label:
                if re.search(r"\d" + name + "I", kernel):
                    yield kernel, body
                kernel, body = label.group(1), []
            elif line.startswith("\t"):
                body.append(line.split("//")[0].strip())


def test_rows_that_are_read_stay_in_the_caches_or_leave_past_them(code_objects):  # noqa: F811
    """Each type and head size in both forms: all stores of rows marked as streaming, or none."""
    forms = []
    for kernel, body in _kernels(code_objects, "cache_read_kernel"):
        stores = [x for x in body if x.startswith("global_store_dwordx4")]
        assert len(stores) == 2 and len([x for x in body if "_store_" in x]) == 2, kernel
        past = [x for x in stores if re.search(r"\bnt\b", x)]
        assert len(past) in (0, 2), stores
        forms.append(len(past))
    assert sorted(forms) == [0] * 6 + [2] * 6, forms
