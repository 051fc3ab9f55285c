"""keep_path_static against its definition (tests/tree_ref.py): bits, and everything else as it was."""
import pytest
import torch

import paper_2511_18191_amd as tsd
from tree_ref import kept

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, N, L, cols, page, H, D, dtype, seed=0, most=20):
    g = torch.Generator().manual_seed(seed)
    n = B * cols + 1
    pools = [torch.randn(L, n, page, H, D, generator=g).to(dtype).cuda() for _ in range(2)]
    table = torch.randperm(n, generator=g)[: B * cols].to(torch.int32).view(B, cols)
    held = torch.randint(0, most + 1, (B,), generator=g).to(torch.int32)
    path = torch.full((B, N), -1, dtype=torch.int32)
    for b in range(B):
        m = int(torch.randint(0, N + 1, (1,), generator=g))
        path[b, :m] = torch.randperm(N, generator=g)[:m].sort().values.to(torch.int32)
    return pools[0], pools[1], table, held, path


def run(k, v, table, held, path, page):
    want = [kept(x.cpu(), table, held, path, page) for x in (k, v)]
    assert tsd.keep_path_static(k, v, table.cuda(), held.cuda(), path.cuda()) is None
    assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,N,L,cols,page,H,D", [
    (1, 1, 1, 2, 16, 1, 8), (1, 4, 1, 2, 16, 8, 128), (5, 26, 3, 4, 16, 2, 64), (3, 64, 2, 90, 1, 3, 40), (2, 65, 1, 6, 16, 4, 80), (2, 200, 2, 8, 32, 1, 256),
    (1, 256, 1, 2, 256, 5, 96), (40, 17, 4, 5, 8, 2, 16), (2, 30, 70, 4, 16, 1, 24)])
def test_sizes(dtype, B, N, L, cols, page, H, D):
    k, v, table, held, path = inputs(B, N, L, cols, page, H, D, dtype)
    run(k, v, table, held, path, page)


def test_a_layer_without_its_dimension():
    k, v, table, held, path = inputs(3, 20, 2, 4, 16, 2, 64, BF)
    run(k[1], v[1], table, held, path, 16)


def test_paths():
    # nothing kept, all kept, ends that are no -1, entries that do not go up, out of range
    B, N, page = 9, 70, 16
    k, v, table, held, path = inputs(B, N, 2, 7, page, 2, 64, FP)
    path[0], path[1], path[2, :4] = -1, torch.arange(N), torch.tensor([0, 3, 3, 9])
    path[3, :5], path[4, :3], path[5, :3] = torch.tensor([2, 5, 4, 8, 9]), torch.tensor([1, N, N + 1]), torch.tensor([3, 2 ** 31 - 1, 5])
    path[6] = torch.arange(N).flip(0)
    path[7, :3] = torch.tensor([-2 ** 31, 4, 5])
    path[8] = torch.cat([torch.arange(0, 69), torch.tensor([69])])
    path[8, 66:] = torch.tensor([67, 68, 69, 70])
    run(k, v, table, held, path, page)


def test_holes_and_slots_beyond_the_table():
    B, N, page = 6, 40, 8
    k, v, table, held, path = inputs(B, N, 2, 8, page, 2, 64, BF)
    path[:] = torch.arange(0, 2 * N, 2).where(torch.arange(N) < N // 2, torch.tensor(-1))
    table[0, 2], table[1, 0], table[2, :], table[3, 3] = -1, 10 ** 6, -1, -2 ** 31
    held[4], held[5] = 60, -3
    run(k, v, table, held, path, page)
    held[:] = torch.tensor([2 ** 31 - 1, 2 ** 30, 2 ** 30 + 1, -2 ** 31, 64, 63])
    run(k, v, table, held, path, page)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_orders_of_caches(dtype):
    # heads outside tokens; keys and values of a page side by side; layers inside pages
    B, N, page, H, D, cols, L = 3, 30, 16, 2, 64, 4, 3
    _, _, table, held, path = inputs(B, N, 1, cols, page, H, D, dtype)
    n = B * cols + 1
    for shape, order, both in (((n, 2, H, page, D), None, 1), ((n, L, 2, page, H, D), None, 2), ((2, L, n, H, page, D), None, 0)):
        whole = torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        k, v = whole.select(both, 0), whole.select(both, 1)
        if both == 1:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        elif both == 2:
            k, v = k.transpose(0, 1), v.transpose(0, 1)
        else:
            k, v = k.transpose(2, 3), v.transpose(2, 3)
        run(k, v, table, held, path, page)


def test_versions_and_inference_mode():
    k, v, table, held, path = inputs(2, 10, 1, 4, 16, 2, 64, FP)
    before = k._version, v._version
    run(k, v, table, held, path, 16)
    assert k._version > before[0] and v._version > before[1]
    with torch.inference_mode():
        k, v, table, held, path = inputs(2, 10, 1, 4, 16, 2, 64, FP)
        run(k, v, table, held, path, 16)


def test_replayed_graphs():
    k, v, table, held, path = inputs(4, 30, 2, 5, 16, 2, 64, BF)
    t, h, p = table.cuda(), held.cuda(), path.cuda()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        tsd.keep_path_static(k, v, t, h, p)
    torch.cuda.synchronize()
    for step in range(4):
        k.normal_()
        v.normal_()
        h.copy_((held + 3 * step) % 30)
        want = [kept(x.cpu(), table, h.cpu(), path, 16) for x in (k, v)]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])


def test_offsets_beyond_32_bits():
    page, H, D = 64, 8, 128
    n = (1 << 32) // (page * H * D) + 40
    if torch.cuda.mem_get_info()[0] < 3 * n * page * H * D * 2:
        pytest.skip("needs some 26 GB of device memory")
    k, v = (torch.empty(n, page, H, D, dtype=BF, device="cuda") for _ in range(2))
    pages = [n - 1, 5, n - 30]
    small = torch.randn(2, len(pages), page, H, D, generator=torch.Generator().manual_seed(4)).to(BF)
    for i, at in enumerate(pages):
        k[at], v[at] = small[0, i].cuda(), small[1, i].cuda()
    held, path = torch.tensor([60], dtype=torch.int32), torch.tensor([[0, 7, 30, 90] + [-1] * 96], dtype=torch.int32)
    tsd.keep_path_static(k, v, torch.tensor([pages], dtype=torch.int32).cuda(), held.cuda(), path.cuda())
    for pool, x in zip((k, v), small):
        want = kept(x, torch.tensor([[0, 1, 2]]), held, path, page)
        assert all(torch.equal(pool[at].cpu(), want[i]) for i, at in enumerate(pages))
