"""The ends where one launch would have 2^32 threads in x or more, which the runtime refuses: the work goes out in several.

Bounds, fixed before the first run: the rows of an embedding with scale 1 are the table's, exactly; a norm's bf16 result is an fp32 value rounded
once, 2^-8 as in the tests of its formula.
"""
import pytest
import torch

import paper_2601_05732_amd as mhcl

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_norm_of_many_short_rows():
    T, C = 2 ** 26 + 3, 8                          # 64 threads a token: 2^32 and some
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(T, 1, C, device="cuda", dtype=BF).normal_(generator=g)
    gain = 1 + 0.1 * torch.randn(C, device="cuda", generator=g)
    h = mhcl.streams_norm(x, gain, eps=1e-5)
    for t0 in range(0, T, 2 ** 23):
        s = x[t0:t0 + 2 ** 23, 0].double()
        want = gain.double() * s / (s.square().mean(dim=1, keepdim=True) + 1e-5).sqrt()
        got = h[t0:t0 + 2 ** 23].double()
        assert bool(((got - want).abs() <= 2 ** -8 * want.abs() + 1e-30).all()), t0


def test_embedding_of_many_tokens():
    T, C, V = 2 ** 24 + 5, 1032, 4099              # 256 threads a token; 35 GB
    g = torch.Generator(device="cuda").manual_seed(2)
    table = torch.empty(V, C, device="cuda", dtype=BF).normal_(generator=g)
    ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g)
    x = mhcl.embed_tokens(table, ids, 1)
    for t0 in range(0, T, 2 ** 21):
        assert torch.equal(x[t0:t0 + 2 ** 21, 0], table[ids[t0:t0 + 2 ** 21].long()]), t0


def test_zeros_of_a_large_table_without_tokens():
    V, C = 2 ** 22 + 1, 1024                       # 2^32 words and some, 17 GB
    d = mhcl.EndsDesc(C, 0, 1, V, BF, F)
    g_table = torch.ones(V, C, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    ws = torch.empty(mhcl.ends_workspace_bytes(d, mhcl.OP_EMBED_BWD), device="cuda", dtype=torch.uint8)
    mhcl.mhcl_embed_bwd(d, none, torch.empty(0, 1, C, device="cuda", dtype=BF), g_table, False, ws)
    for v0 in range(0, V, 2 ** 19):
        assert not g_table[v0:v0 + 2 ** 19].any(), v0
