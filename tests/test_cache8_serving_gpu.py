"""The 8-bit cache in use: pages and lengths of a serving step, norm and rotation, writing, attention, drops, the accepted path of a tree; captured
and replayed; on streams."""
import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib
from test_cache8_gpu import check_attention, filled, i32, new_cache, on_gpu, same_bytes

pytestmark = pytest.mark.gpu


class Serving:
    def __init__(self, dtype, B=3, H=8, Hkv=2, D=128, R=64, M=8):
        self.dtype, self.B, self.H, self.Hkv, self.D, self.R, self.M = dtype, B, H, Hkv, D, R, M
        self.host = new_cache(B * M, Hkv, R, D, seed=11)
        self.dev = on_gpu(self.host)
        g = torch.Generator().manual_seed(5)
        self.table, self.free = torch.full((B, M), -1, dtype=torch.int32, device="cuda"), torch.randperm(B * M, generator=g).to(torch.int32).cuda()
        self.pool, self.lens = i32([B * M, 0]), i32([0] * B)
        self.inv = (10000.0 ** (-torch.arange(D // 2).double() / (D // 2))).float().cuda()
        self.w = [(1 + 0.1 * torch.randn(D, generator=g)).to(dtype).cuda() for _ in range(2)]

    def project(self, S, seed):
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(self.B, S, (self.H + 2 * self.Hkv) * self.D, generator=g).to(self.dtype).cuda()
        q, k, v = x.split([self.H * self.D, self.Hkv * self.D, self.Hkv * self.D], dim=-1)
        return q.view(self.B, S, self.H, self.D), k.view(self.B, S, self.Hkv, self.D), v.view(self.B, S, self.Hkv, self.D)

    def append(self, counts, S, seed, depths=None):
        """A step's tokens into the cache; (queries, slots)."""
        q, k, v = self.project(S, seed)
        before = self.lens
        self.lens, slots, positions, self.pool = lib.cache_step(before, i32(counts), S, self.R, pages=(self.table, self.free, self.pool), depths=depths)
        assert int(self.pool[1]) == 0
        qr, kr = lib.qk_norm_rope(q, k, *self.w, positions, self.inv)
        self.write(kr.transpose(1, 2), v, before, self.lens)
        return qr, slots

    def write(self, k, v, old, new):
        lib.cache8_write(k, v, *self.dev, old, new, block_table=self.table)
        for x, codes, scales in ((k, self.host[0], self.host[2]), (v, self.host[1], self.host[3])):
            ref.write(x.cpu(), codes, scales, old.tolist(), new.tolist(), self.table.cpu())
        same_bytes(self.dev, self.host)

    def attend(self, q):
        return check_attention(q, self.host, self.dev, self.lens.tolist(), self.table.cpu(), self.M * self.R, causal=True)

    def drop(self, counts):
        self.lens, _, _, self.pool = lib.cache_step(self.lens, i32(counts), 1, self.R, pages=(self.table, self.free, self.pool))
        assert int(self.pool[1]) == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_steps(dtype):
    """Prefill, decoding, drafts in a chain of which some are rejected, a request that ends and another that takes its pages."""
    s = Serving(dtype)
    s.attend(s.append([150, 5, 63], 150, 1)[0])
    for i in range(3):
        s.attend(s.append([1, 1, 1], 1, 10 + i)[0])
    s.attend(s.append([6, 6, 6], 6, 20)[0])
    s.drop([-2, -6, -5])
    s.attend(s.append([1, 1, 1], 1, 21)[0])
    s.drop([0, 0, -int(s.lens[2])])
    s.attend(s.append([1, 1, 90], 90, 22)[0])
    s.attend(s.append([0, 1, 1], 1, 23)[0])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_the_accepted_path_of_a_tree(dtype):
    """Tokens of a tree are appended; the accepted ones, a path that is no prefix, are read, the tree is dropped, and they are written in its place."""
    s = Serving(dtype)
    s.append([150, 5, 63], 150, 1)
    T, paths = 7, [[0, 2, 5], [1], [3, 4, 6]]
    base = s.lens
    _, slots = s.append([T] * 3, T, 2)
    src = torch.tensor([[0] * (T - len(p)) + p for p in paths], device="cuda")                # the path at the end of an entry's row
    k, v = lib.cache8_read(*s.dev, slots.gather(1, src), dtype)
    for x, codes, scales in ((k, s.host[0], s.host[2]), (v, s.host[1], s.host[3])):
        values = ref.values(codes, scales).transpose(1, 2).flatten(0, 1)[slots.gather(1, src).long().cpu()].transpose(1, 2)
        assert torch.equal(x.cpu().double(), values)
    s.drop([len(p) - T for p in paths])
    s.write(k.transpose(1, 2), v.transpose(1, 2), base, s.lens)
    assert s.lens.tolist() == [n + len(p) for n, p in zip(base.tolist(), paths)]
    s.attend(s.append([1, 1, 1], 1, 3)[0])


def test_a_refused_step_writes_nothing():
    s = Serving(torch.bfloat16, M=2)
    s.append([100, 5, 63], 100, 1)
    q, k, v = s.project(60, 2)
    new, _, _, pool = lib.cache_step(s.lens, i32([60, 1, 1]), 60, s.R, pages=(s.table, s.free, s.pool))
    assert int(pool[1]) != 0
    lib.cache8_write(k, v, *s.dev, s.lens, new, block_table=s.table)
    same_bytes(s.dev, s.host)


@pytest.mark.parametrize("Sq", [1, 5, 40])
def test_captured_and_replayed(Sq):
    """A step in a graph: replayed on other tokens and lengths, with eager work between the replays, each against the same calls made eagerly."""
    B, H, Hkv, D, cap = 3, 8, 2, 64, 1500
    dev = on_gpu(new_cache(B, Hkv, cap, D, seed=1))
    first = [x.clone() for x in (dev[0].view(torch.uint8), dev[1].view(torch.uint8), dev[2], dev[3])]
    old, new = i32([0] * B), i32([1] * B)
    k, v = (torch.zeros(B, Sq, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(B, H, Sq, D, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(B, 4, dtype=torch.int32, device="cuda")

    def step():
        lib.cache8_write(k, v, *dev, old, new)
        o, lse = lib.sdpa_kv8(q, *dev, causal=True, kv_lens=new, return_lse=True)
        return (o, lse) + lib.cache8_read(*dev, slots, torch.float16)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for turn, lens in enumerate([[0, 700, 31], [900, 1400, 1], [64, 1459, 500], [3, 2, 1]]):
        def inputs():
            for x, y in zip((dev[0].view(torch.uint8), dev[1].view(torch.uint8), dev[2], dev[3]), first):
                x.copy_(y)
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(turn)).to(x.dtype))
            old.copy_(i32(lens))
            new.copy_(i32([n + Sq for n in lens]))
            slots.copy_(i32([[b * cap + x for x in (0, lens[b], lens[b] + Sq - 1, cap - 1)] for b in range(B)]))
        inputs()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in captured] + [x.clone() for x in (dev[0].view(torch.uint8), dev[1].view(torch.uint8), dev[2], dev[3])]
        inputs()
        want = list(step()) + [dev[0].view(torch.uint8), dev[1].view(torch.uint8), dev[2], dev[3]]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            same = (a == b) | ((a != a) & (b != b))
            assert same.all()


def test_streams_at_once():
    """Calls on two streams at the same time, each with its own results; the cache is read by both."""
    lens = [9000, 3000]
    host, dev, _ = filled(2, 2, 9000, 64, lens, 0, seed=6)
    qs = [torch.randn(2, 8, Sq, 64, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda() for Sq in (1, 3, 30, 1, 3, 30)]
    want = [lib.sdpa_kv8(q, *dev, causal=True, kv_lens=i32(lens)) for q in qs]
    torch.cuda.synchronize()
    streams, got, n = [torch.cuda.Stream() for _ in range(2)], [], i32(lens)
    torch.cuda.synchronize()
    for i, q in enumerate(qs * 3):
        with torch.cuda.stream(streams[i % 2]):
            got.append(lib.sdpa_kv8(q, *dev, causal=True, kv_lens=n))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i % len(qs)]) for i, a in enumerate(got))


def test_tensor_arguments_are_checked():
    host = new_cache(2, 2, 64, 64)
    k, v, ks, vs = on_gpu(host)
    q = torch.zeros(2, 4, 1, 64, dtype=torch.float16, device="cuda")
    x = torch.zeros(2, 3, 2, 64, dtype=torch.float16, device="cuda")
    n, table, slots = i32([3, 3]), i32([[0], [1]]), i32([[0, 1], [2, 3]])
    refused = [
        lambda: lib.sdpa_kv8(q, k.view(torch.uint8), v, ks, vs), lambda: lib.sdpa_kv8(q, k, v, ks[:1], vs), lambda: lib.sdpa_kv8(q, k, v, ks.int(), vs),
        lambda: lib.sdpa_kv8(q, k.transpose(1, 2), v, ks, vs), lambda: lib.sdpa_kv8(q, k, v[:, :1], ks, vs), lambda: lib.sdpa_kv8(q.float(), k, v, ks, vs),
        lambda: lib.sdpa_kv8(q[:1], k, v, ks, vs), lambda: lib.sdpa_kv8(q[:, :3].contiguous(), k, v, ks, vs), lambda: lib.sdpa_kv8(q, k, v, ks, vs, kv_lens=n.long()),
        lambda: lib.sdpa_kv8(q, k, v, ks, vs, kv_lens=n.cpu()), lambda: lib.sdpa_kv8(q, k, v, ks, vs, out=q.float()),
        lambda: lib.sdpa_paged8(q, k, v, ks, vs, n, table.cpu()), lambda: lib.sdpa_paged8(q, k, v, ks, vs, None, table), lambda: lib.sdpa_paged8(q, k, v, ks, vs, n, table[:1]),
        lambda: lib.cache8_write(x, x[:, :2], k, v, ks, vs, n, n), lambda: lib.cache8_write(x, x.bfloat16(), k, v, ks, vs, n, n), lambda: lib.cache8_write(x.float(), x.float(), k, v, ks, vs, n, n),
        lambda: lib.cache8_write(x[..., ::2], x[..., ::2], k, v, ks, vs, n, n), lambda: lib.cache8_write(x, x, k, v, ks, vs, n, n[:1]), lambda: lib.cache8_write(x, x, k, k, ks, vs, n, n),
        lambda: lib.cache8_write(x, x, k, v, ks, ks, n, n), lambda: lib.cache8_write(x, x, k, v, ks, vs, ks.view(-1).view(torch.int32)[:2], n),
        lambda: lib.cache8_read(k, v, ks, vs, slots, torch.float32), lambda: lib.cache8_read(k, v, ks, vs, slots, "float16"), lambda: lib.cache8_read(k, v, ks, vs, slots[0], torch.float16),
        lambda: lib.cache8_read(k, v, ks, vs, slots, torch.float16, out=(x, x)),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, lib.TiledSdpaError)):
            call()
            pytest.fail(f"call {i} was not refused")
    with pytest.raises(lib.TiledSdpaError):
        lib.sdpa_paged8(q, *on_gpu(new_cache(2, 2, 48, 64)), n, table)
    k, v, ks, vs = on_gpu(host)
    a = lib.sdpa_kv8(q + 1, k, v, ks, vs, kv_lens=n)
    b = lib.sdpa_kv8(q + 1, k, v, ks.view(torch.float8_e8m0fnu), vs.view(torch.float8_e8m0fnu), kv_lens=n)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    empty = lib.sdpa_kv8(q[:, :, :0], k, v, ks, vs)
    assert empty.shape == (2, 4, 0, 64)
    assert lib.cache8_read(k, v, ks, vs, slots[:, :0], torch.float16)[0].shape == (2, 2, 0, 64)
    lib.cache8_write(x[:, :0], x[:, :0], k, v, ks, vs, n, n)
    same_bytes((k, v, ks, vs), host)


def test_results_in_what_the_call_reads_are_refused():
    k, v, ks, vs = on_gpu(new_cache(2, 2, 2048, 64))
    q = torch.zeros(2, 4, 1, 64, dtype=torch.float16, device="cuda")
    n, table, p8 = i32([2000, 3]), i32([[0], [1]]), tuple(on_gpu(new_cache(2, 2, 2048, 64)))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    inside = ws[:q.numel() * 2].view(torch.float16).view(q.shape)
    of_k = k.view(torch.uint8).view(-1)[:q.numel() * 2].view(torch.float16).view(q.shape)
    for call in (lambda: lib.sdpa_kv8(q, k, v, ks, vs, kv_lens=n, out=q), lambda: lib.sdpa_kv8(q, k, v, ks, vs, out=of_k), lambda: lib.sdpa_kv8(q, k, v, ks, vs, workspace=v.view(torch.uint8)),
                 lambda: lib.sdpa_kv8(q, k, v, ks, vs, out=inside, workspace=ws), lambda: lib.sdpa_kv8(q, k, v, ks, vs, workspace=ks),
                 lambda: lib.sdpa_paged8(q, *p8, n, table, workspace=table.view(torch.uint8)), lambda: lib.sdpa_paged8(q, *p8, n, table, workspace=n.view(torch.uint8))):
        with pytest.raises(ValueError, match="overlap"):
            call()
    want = lib.sdpa_kv8(q + 1, k, v, ks, vs, kv_lens=n)
    out = torch.empty_like(q)
    assert lib.sdpa_kv8(q + 1, k, v, ks, vs, kv_lens=n, out=out, workspace=ws) is out and torch.equal(out.view(torch.int16), want.view(torch.int16))
