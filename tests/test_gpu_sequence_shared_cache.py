"""Sequences that read the same cache: more than 2^31 units of 64 keys in all."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_many_sequences_over_one_long_cache():
    """Each query has one key of its own that outweighs all others by exp(32): its value is the result.  The keys are
    signs of 8 bits, -16 or 16 for queries of 1 / 4: scores 32 for the own key, 24 and less for those of other bits, and
    0 for the other 1.4e8 keys, whose values are 0.  The weights beside the own one's add up to less than 1.4e8 exp(-32) + 8
    exp(-8) + ... < 5e-3 of it, which the queries' order of values keeps apart."""
    from paper_2402_09633_gb300 import WindowAttention
    seqs, n, D, codes = 1024, 2 ** 27 + 2 ** 20, 8, 256
    bits = torch.tensor([[1.0 if c >> i & 1 else -1.0 for i in range(D)] for c in range(codes)])
    rows = torch.arange(codes) * (n // codes) + torch.randint(0, n // codes, (codes,), generator=torch.Generator().manual_seed(0))
    rows[0], rows[-1] = 0, n - 1
    k, v = (torch.zeros(n, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[rows.cuda(), 0] = (16 * bits).bfloat16().cuda()
    v[rows.cuda(), 0] = bits.bfloat16().cuda()
    own = torch.arange(seqs) % codes
    q = (bits[own] / 4)[:, None].bfloat16().cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
    att = WindowAttention()
    out = att(q, k, v, i32(range(seqs + 1)), right=0, scale=1.0, kv_start=i32([0] * seqs), kv_len=i32([n] * seqs), max_q=1,
              max_kv=n)
    assert att.status() == 0
    # a sign that another key's value has the other way round weighs twice; and one rounding to bf16
    assert float((out[:, 0].float().cpu() - bits[own]).abs().max()) <= 2 * 5e-3 + 2.0 ** -8
