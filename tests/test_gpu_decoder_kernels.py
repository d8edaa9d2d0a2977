"""Every kernel that the decoder's projection and cache choose by size, against the definition in binary64.  Which shape reaches which kernel is checked in
test_decoder_rules.py."""
import pytest

pytestmark = pytest.mark.gpu

import torch  # noqa: E402

from test_gpu_decoder import BF16, F16, P, Plan, check_linear, gen, offsets, quantised, weights  # noqa: E402, F401

# tile, stages in flight, M, N, K
TILED = [(0, 4, 70, 1296, 960), (0, 4, 150, 1552, 576), (0, 4, 300, 144, 704), (0, 2, 33, 528, 448), (0, 2, 300, 80, 192),
         (1, 4, 533, 1296, 576), (1, 4, 300, 2064, 704), (1, 2, 533, 1296, 448), (1, 2, 700, 1552, 832), (1, 2, 150, 4112, 960), (1, 2, 600, 1024, 128),
         (2, 4, 533, 2512, 1600), (2, 4, 700, 2064, 704), (2, 2, 1000, 1552, 832), (2, 2, 3000, 528, 320), (2, 2, 3000, 528, 192),
         (3, 2, 1500, 2512, 448), (3, 2, 1000, 2064, 704), (3, 2, 2100, 1296, 320), (3, 2, 700, 4112, 192), (3, 2, 1500, 4112, 1024),
         (4, 2, 1000, 4112, 448), (4, 2, 2100, 2064, 704), (4, 2, 3000, 1552, 320), (4, 2, 2100, 4112, 576), (4, 2, 2100, 2512, 64)]
# M, N, K
FEW = [(1, 4112, 8192), (1, 4080, 8192), (2, 4112, 1024), (9, 2064, 1984), (16, 4112, 960), (11, 4128, 2048), (8, 4112, 4096), (3, 80, 2112), (5, 272, 3328), (16, 528, 1984),
       (2, 96, 6208), (5, 272, 8192), (6, 2064, 8192), (9, 80, 4672), (13, 2064, 4160), (16, 528, 3328), (8, 1040, 2048), (3, 16, 1024), (4, 144, 576),
       (16, 272, 4096), (7, 80, 8192), (16, 4112, 8128), (1, 1040, 8256), (12, 80, 14336)]
# contexts, how many of their positions are new, key heads, head_dim, page_len: more than 32768 rows of a head each, written and read
CACHES = [([4000, 0, 17, 600], [3900, 0, 17, 600], 8, 128, 64), ([3001, 1, 700, 65], [2800, 1, 33, 65], 12, 64, 16), ([11000, 23000], [10999, 22011], 1, 128, 256)]


def run_linear(P, M, N, K, dtype, bias, gelu):
    x = torch.randn(M, K, generator=gen(M * 7 + K)).to(dtype)
    W, s_w = weights(N, K, N)
    b = torch.randn(N, generator=gen(5)) if bias else None
    Wp = P.pack_weight_i8(W.cuda())
    dev = [t if t is None else t.cuda() for t in (s_w, b)]
    y = P.linear_i8_tokens(x.cuda(), Wp, *dev, gelu)
    codes, steps = P.quantize_tokens(x.cuda())
    assert torch.equal(y, P.gemm_i8_tokens_packed(codes, steps, Wp, *dev, gelu, dtype))
    check_linear(y, *quantised(x), W, s_w, b, gelu, dtype)


@pytest.mark.parametrize("tile,depth,M,N,K", TILED)
def test_linear_of_many_rows(P, tile, depth, M, N, K):
    run_linear(P, M, N, K, F16 if (M + N) % 32 else BF16, K % 128 == 0, False)
    run_linear(P, M, N, K, BF16 if (M + N) % 32 else F16, K % 128 != 0, True)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N,K", FEW)
def test_linear_of_few_rows(P, M, N, K, dtype):
    run_linear(P, M, N, K, dtype, M % 2 == 0, M % 3 == 0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,new,G,D,page", CACHES)
def test_cache_of_many_rows(P, lens, new, G, D, page, dtype):
    plan = Plan(P, lens, new, G, D, page, seed=G)
    before = plan.fill(P, dtype, 4)
    k, v = (torch.randn(plan.total + 2, G, D, generator=gen(i)).to(dtype) for i in (7, 8))   # two rows behind the last sequence
    idle = sorted(set(range(plan.cache.pages)) - {p for t in plan.tables for p in t})
    held = [t[idle].clone() for t in (plan.cache.k, plan.cache.v)]
    P.cache_write(plan.cache, k.cuda(), v.cuda(), *plan.args, max(new))
    out = tuple(torch.full((sum(lens) + 3, G, D), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    P.cache_read(plan.cache, plan.args[0], offsets(lens).cuda(), plan.args[2], max(lens), sum(lens) + 3, dtype, out=out)
    for i, (got, x) in enumerate(zip(out, (k, v))):
        want, at = [], 0
        for b, (n, m) in enumerate(zip(lens, new)):
            c, s = quantised(x[at:at + m])
            want.append(torch.cat([before[b][i][: n - m], c * s[..., None]]))
            at += m
        assert torch.equal(got[: sum(lens)].cpu(), torch.cat(want).float().to(dtype))
        assert (got[sum(lens):] == 9).all()
    assert torch.equal(plan.cache.k[idle], held[0]) and torch.equal(plan.cache.v[idle], held[1])
