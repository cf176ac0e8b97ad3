"""The pages of a cache step as any sequence of three tensors, one whose tensors nobody else holds among them."""
import pytest
import torch

from test_cache_index_gpu import i32, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def test_pages_that_only_the_argument_holds(lib):  # noqa: F811
    """The step reads and writes them until it ends, so that its results are not put into their memory."""
    B, M, R, S = 40, 64, 16, 300
    lens, counts = i32([0] * B), i32([S - b for b in range(B)])
    own = [torch.full((B, M), -1, dtype=torch.int32, device="cuda"), torch.randperm(B * M, device="cuda").to(torch.int32), i32([B * M, 0])]
    for pages in (lambda: (t.clone() for t in own), lambda: [t.clone() for t in own], lambda: iter([own[0].clone(), own[1].clone(), own[2].clone()])):
        for _ in range(3):
            got = lib.cache_step(lens, counts, S, R, pages=pages())
            mine = [t.clone() for t in own]
            want = lib.cache_step(lens, counts, S, R, pages=mine)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            spans = sorted((t.data_ptr(), t.numel() * 4) for t in got)
            assert all(a + n <= b for (a, n), (b, _) in zip(spans, spans[1:]))
