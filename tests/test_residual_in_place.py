"""A residual may be the result's own rows (include/aiq.h), so no kernel with a residual may promise the compiler that what it writes is not read by
another name (no GPU needed: the sources are read)."""
import os
import re

from test_chain_memory_rule import CSRC, _kernels


def test_no_kernel_with_a_residual_has_restrict_on_what_it_writes():
    seen = set()
    for name in sorted(os.listdir(CSRC)):
        if not (name.startswith("mx") or name == "experts.cu") or not name.endswith((".cu", ".cuh")):
            continue
        for kernel, params, body in _kernels(re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())):
            if not re.search(r"\bresidual\b", params + body):
                continue
            seen.add(kernel)
            for p in re.findall(r"(\w+)\s*\*\s*__restrict__\s+(\w+)", params):
                assert re.search(r"const\s+%s\s*\*\s*__restrict__\s+%s\b" % p, params), f"{name}: {kernel} writes {p[1]} as __restrict__"
                assert p[1] != "residual", f"{name}: {kernel}"
    assert seen >= {"mx_tc_kernel", "mx_few_kernel", "mx_product_rows_kernel", "mx_product_row_kernel", "combine_kernel"}
