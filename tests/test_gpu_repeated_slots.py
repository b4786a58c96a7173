"""Rows with one slot on the GPU: ssd_rope_kv leaves the last of them in calls of up to 129 rows; else any may stay."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ssd():
    import paper_2309_08168_gb300 as m
    return m


@pytest.mark.parametrize("typ", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,places", [(2, 1), (4, 2), (40, 3), (128, 1), (129, 1), (129, 60)])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (64, 8)])
def test_the_last_row_of_a_slot_stays(ssd, typ, n, places, heads, kv_heads):
    g = torch.Generator().manual_seed(n + places)
    q, k, v = (torch.randn(n, h, 64, generator=g).to(typ).cuda() for h in (heads, kv_heads, kv_heads))
    at = torch.randint(0, places, (n,), generator=g).int()
    at[n // 2] = -1 if n > 4 else at[n // 2]
    last = {int(s): i for i, s in enumerate(at) if s >= 0}
    c = torch.bfloat16 if typ is torch.bfloat16 else torch.float16
    pages = places // 16 + 1
    rope, pos = ssd.ssd_rope_init(64), torch.arange(n, dtype=torch.int32, device="cuda")

    def caches():
        return [torch.zeros(1, pages, kv_heads, 16, 64, dtype=c, device="cuda") for _ in range(2)]

    def run(cache, slots):
        out = torch.empty_like(q)
        ssd.ssd_rope_kv(ssd.PagedKV(*cache), 0, rope, q, k, v, pos, slots.cuda(), out, cuda_stream=torch.cuda.current_stream().cuda_stream)
        return out
    only = torch.full_like(at, -1)  # the same with the last rows' slots alone
    for s, i in last.items():
        only[i] = s
    want = caches()
    out = run(want, only)
    for _ in range(5):
        got = caches()
        assert torch.equal(run(got, at), out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()


@pytest.mark.parametrize("normed", [False, True])
def test_other_rows_of_larger_calls(ssd, normed):
    """The rows with slots of their own are right."""
    n = 400
    k, v = (torch.randn(n, 2, 64, device="cuda").half() for _ in range(2))
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    slots[7::50] = 7
    cache = [torch.zeros(1, 25, 2, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    call = ssd.ssd_norm_rope_kv if normed else ssd.ssd_rope_kv
    call(ssd.PagedKV(*cache), 0, ssd.ssd_rope_init(64), k, k, v, slots, slots, torch.empty_like(k), cuda_stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    rows = cache[1][0].transpose(1, 2).reshape(-1, 2, 64)
    own = torch.ones(n, dtype=torch.bool, device="cuda")
    own[7::50] = False
    assert torch.equal(rows[:n][own], v[own]) and (rows[57:n:50] == 0).all()
    assert all(any(torch.equal(rows[7, h], v[r, h]) for r in range(7, n, 50)) for h in range(2))
