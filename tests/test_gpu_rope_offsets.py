"""Rotary positions on heads whose elements lie more than 2^32 bytes, and 2^31 elements, apart."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

TOKENS, HD, PITCH = 40, 64, 1 << 26  # 2.7e9 elements of 2 bytes


@pytest.fixture(scope="module")
def ress():
    import paper_2609_35593_gb300 as r
    return r


def far(heads, by_token):
    """[TOKENS, heads, HD] with its tokens, or its heads, PITCH elements apart."""
    n, inner = (TOKENS, heads * HD) if by_token else (heads, TOKENS * HD)
    strides = (PITCH, HD, 1) if by_token else (HD, PITCH, 1)
    return torch.zeros((n - 1) * PITCH + inner, device="cuda", dtype=torch.bfloat16).as_strided((TOKENS, heads, HD), strides)


@pytest.mark.parametrize("heads,by_token", [(1, True), (3, True), (16, True), (40, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_far_heads_as_near_ones(ress, heads, by_token, norm):
    g = torch.Generator(device="cuda").manual_seed(heads)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32).bfloat16()
    plan = ress.rope_plan((32, 32))
    pos = torch.randint(0, 37, (TOKENS, 2), generator=g, device="cuda", dtype=torch.int32)
    x, dy = normal(TOKENS, heads, HD), normal(TOKENS, heads, HD)
    params = (normal(HD).float(), normal(HD).float()) if norm else None
    results = []
    for make in (lambda: torch.empty_like(x), lambda: far(heads, by_token)):
        a, y, d, dx = make(), make(), make(), make()
        a.copy_(x), d.copy_(dy)
        grads = torch.empty(2, HD, device="cuda", dtype=torch.float32)
        ws = torch.empty(ress.rope_workspace_bytes(plan, TOKENS, heads), dtype=torch.uint8, device="cuda")
        ress.rope(plan, pos, a, y, q_norm=params)
        ress.rope_bwd(plan, pos, d, dx, q=a if norm else None, q_norm=params,
                      q_norm_grads=tuple(grads.unbind()) if norm else None, ws=ws)
        results.append([y.contiguous(), dx.contiguous()] + ([grads] if norm else []))
        del a, y, d, dx
        torch.cuda.empty_cache()
    assert all(torch.equal(p, q) for p, q in zip(*results))
    assert bool(results[0][0].isfinite().all()) and bool(results[0][0].any())
