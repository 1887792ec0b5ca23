"""The instances of the row kernels that are built are those that a launch can take."""
import os
import re
import subprocess

from test_kernel_listing import LLVM, code_objects  # noqa: F401


def test_four_vectors_a_thread_of_256_only_with_alternatives(code_objects):  # noqa: F811
    """cut_rows() cuts rows without alternatives into chunks of two or eight vectors a thread."""
    names = set()
    for f in code_objects:
        table = subprocess.check_output([os.path.join(LLVM, "llvm-readelf"), "--symbols", "--wide", f], text=True)
        names |= set(re.findall(r"(\S*logprobs_kernelI\S+E)\S*", table))
    found = {re.search(r"ILi(\d)ELi(\d+)ELi(\d)ELb([01])ELb([01])E", n).groups() for n in names if "logprobs_kernelI" in n}
    assert {(t, "256", "4", "1", e) for t in "0123" for e in "01"} <= found
    assert not any(threads == "256" and vecs == "4" and top == "0" for _, threads, vecs, top, _ in found)
