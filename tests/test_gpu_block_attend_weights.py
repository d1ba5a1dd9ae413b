"""How exactly 16-bit attention weighs: values that cancel, so that what comes out is small and its own rounding does not hide that of the weights."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu
LOST = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -22 + 2.0 ** -30 * 64}       # of a weight: of 64 places, none below a 64th here


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("places", [2, 5, 16, 23, 50])
@pytest.mark.parametrize("news", [1, 9])
def test_values_that_cancel(news, places, D, dtype):
    import paper_2102_05187_amd as comet
    g = torch.Generator().manual_seed(places + D)
    G, block, n = 4, 16, places + news - 1
    M = -(-n // block)
    K, V = torch.zeros((M, block, 1, D)), torch.zeros((M, block, 1, D))
    key, value = K.view(-1, D), V.view(-1, D)
    key[:n, 0] = torch.rand(n, generator=g)
    value[:n] = torch.randn((n, D), generator=g)
    K = K.to(dtype)
    # the last token reads all of it: its values cancel, as far as the type goes
    w = torch.softmax(K.view(-1, D)[:n, 0].double(), 0)
    most = int(w.argmax())
    x = value[:n].to(dtype).double()
    x[most] = 0
    value[most] = (-(w @ x) / w[most]).float()
    V = V.to(dtype)
    q = torch.zeros((news, G, D))
    q[:, :, 0] = 1
    table = torch.arange(M, dtype=torch.int32)[None]
    sel = torch.arange(M, dtype=torch.int32).expand(news, 1, M).contiguous()
    out, _ = comet.comet_block_attend(q.to(dtype).cuda(), K.cuda(), V.cuda(), table.cuda(), torch.tensor([0, news], dtype=torch.int32).cuda(),
                                      torch.tensor([n], dtype=torch.int32).cuda(), sel.cuda(), scale=1.0)
    v = V.view(-1, D)[:n].double()
    want, mass = w @ v, w @ v.abs()
    # a score is one product in 32 bits, below 2 with its factor: 2^-22 for that, the factor, the maximum and the difference; exp2 2^-22; all that twice, as the sum
    # of weights has it too; sums of `places` terms and those of the wavefronts; the result's own rounding
    weight = LOST[dtype] + 4 * 2.0 ** -22 + 2.0 ** -24 * (n + 64)
    bound = weight * mass * 1.01 + ref.UNIT[dtype] * want.abs() * 1.01 + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert bool(((out[-1].double().cpu() - want).abs() <= bound).all())
