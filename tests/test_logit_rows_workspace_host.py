"""Sizes of the workspaces of the operators on rows of class logits: one for a batch serves every smaller batch."""
import ctypes as C

import pytest

import paper_2108_09413_amd as isr


def _of(size, classes, kind, rows):
    return [size(C.byref(isr.Logits(1 << 40, kind, classes, n, classes, 1.0))) for n in rows]


ROWS = [*range(1, 1100), 1500, 2047, 2048, 4096, 100000, 1 << 22, (1 << 22) + 1, (1 << 31) - 1]


@pytest.mark.parametrize("kind", [isr.F32, isr.BF16])
@pytest.mark.parametrize("classes", [10, 257, 1025, 8193, 16385, 20011, 32000, 32768, 50021, 65536, 65544, 100003, 131072, 262144, 300007, 1 << 24])
def test_the_size_does_not_fall_with_more_rows(kind, classes):
    L = isr.lib()
    for top in (0, 1, 20, 32, 33, 64, 128):
        top = min(top, classes)
        sizes = _of(lambda l: L.isr_logprobs_workspace_bytes(l, top), classes, kind, ROWS)
        assert sizes == sorted(sizes), (classes, top)
    for top, rest in ((1, 0), (128, 1)):
        t = isr.Teacher(1 << 41, 1 << 42, isr.F32, top, 1.0, rest)
        sizes = _of(lambda l: L.isr_distill_workspace_bytes(l, C.byref(t)), classes, kind, ROWS)
        assert sizes == sorted(sizes), (classes, top, rest)


def test_the_size_is_what_the_largest_of_the_smaller_calls_needs():
    """1023 rows of 32000 bf16 in two chunks each, 20 alternatives: 16 bytes a chunk and a list of 128 candidates of 8 bytes."""
    L = isr.lib()
    size = lambda rows: _of(lambda l: L.isr_logprobs_workspace_bytes(l, 20), 32000, isr.BF16, [rows])[0]
    chunks = 2
    most = (1023 * chunks * 16 + 255) // 256 * 256 + 1023 * chunks * 128 * 8
    assert size(1023) == size(1024) == size(1 << 20) == most and size(512) == 0
