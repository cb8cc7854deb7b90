"""How exactly ntp_attn_chunk_shard's softmax weights go into the product with the values, on a real MI355X.

Sequences of up to 32 rows (new tokens x query heads of a KV head): a weight p is multiplied as its bf16 rounding and what that leaves, rounded to bf16 too, so that 2^-8 * 2^-8 = 1.6e-5 of it
is lost at most, whatever else the batch holds.  With the scores' fp32 error, at most 2e-4 of a weight (|score| <= 30, as test_gpu_attn_chunk.py derives it), and the additions' 2^-24 each over
at most 2000 tokens (1.2e-4) that is below 4e-4 of sum p |V| / sum p; besides, half a step of bf16 for the result, 2^-8 |C|."""
import numpy as np
import pytest

from oracle import block_oracle as B
from tests.test_gpu_attn_chunk import BF, F32, Case, _say, f64

pytestmark = pytest.mark.gpu


def _check_few(c, C, few):
    """The rows of the sequences `few`, without the half step of bf16 for their weights."""
    want, _, size, _ = B.attn_chunk(f64(c.Q), *c.numbers, c.starts, c.table.cpu().numpy(), c.lengths, c.max_new, c.max_len, c.plan["q_off"], c.plan["kv_off"], c.group)
    starts = range(c.M + 1) if c.starts is None else c.starts
    rows = np.concatenate([np.arange(starts[s], starts[s + 1]) for s in few])
    over = (np.abs(f64(C) - want) - BF * np.abs(want) - F32 * size)[rows]
    assert (over <= 0).all(), f"{over.max()} over, {(over > 0).sum()} of {over.size} wrong, first {np.argwhere(~(over <= 0))[0]}"


MIXES = [
    # new tokens, lengths, q, kv, d, group, sequences of up to 32 rows
    ([1] * 5, [700, 3, 64, 257, 2000], 3, 1, 128, 3, range(5)),                            # up to 16 rows
    ([4, 2, 1, 5], [700, 33, 64, 900], 8, 2, 64, 4, range(4)),                             # 17 to 32 rows
    ([1] * 3, [500, 1000, 1999], 20, 1, 128, 20, range(3)),                                # one token, 20 query heads
    ([4] * 6, [4, 5, 64, 65, 257, 1023], 8, 1, 128, 8, range(6)),
    ([1, 200, 1, 3, 1], [900, 700, 130, 2000, 30], 4, 2, 128, 2, (0, 2, 3, 4)),            # beside a chunk
    ([1, 1, 300, 2], [77, 1500, 300, 640], 11, 4, 64, 3, (0, 1, 3)),
]


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("news,lengths,q,kv,d,group,few", MIXES)
def test_few_rows_keep_their_weights(news, lengths, q, kv, d, group, few, workspace, fmt):
    """Many nearly equal weights half a step of bf16 off, all to the same side, against values that cancel: without the weights' rest an output is 1.3e-3 off where 3e-4 is allowed.  Every other
    key is 0 and the others k; a query's product with k makes their weight w = (8 + j % 8) / 16 + 2^-9 relative to the zeros', and column j holds values 1 and -(8 + j % 8) / 16."""
    import torch
    _say(f"weights of {news} of {lengths}, {q} query heads on {kv} KV heads of {d}, {fmt} bits, workspace {workspace}")
    c = Case(news, lengths, q, kv, d, 32, 0, 0, group, fmt, seed=d + q)
    odd = torch.arange(32, device="cuda") % 2 == 1
    steps = (8 + torch.arange(d, device="cuda") % 8) / 16
    k = torch.zeros(32, d, device="cuda")
    k[odd, :3] = 1.0
    v = torch.where(odd[:, None], torch.ones(d, device="cuda"), -steps)
    if fmt == 16:
        for t, x in ((c.K, k), (c.V, v)):
            t.copy_(torch.where(t.isnan(), t, x.bfloat16()))
        c.numbers = f64(c.K), f64(c.V)
    else:
        c.numbers = []
        for num, e, x in ((c.raw[0], c.raw[1], k), (c.raw[2], c.raw[3], v)):
            gone = num.float().isnan()
            num.copy_(torch.where(gone, num.float(), x).to(torch.float8_e4m3fn))
            e.copy_(torch.where(gone.any(-1), e, torch.full_like(e, 127)))
            c.numbers.append(np.ldexp(f64(num), (e.cpu().numpy().astype(np.int64) - 127)[..., None]))
    # the score's three bf16 pieces, exact to 2^-24 of it
    score = torch.log((8 + torch.arange(q, device="cuda").double() % 8) / 16 + 2.0 ** -9) * d ** 0.5
    c.Q.zero_()
    Q = c.Q.view(c.M, q, d) if c.Q.is_contiguous() else c.Q.unflatten(1, (q, d))
    for i in range(3):
        part = score.to(torch.bfloat16)
        Q[:, :, i] = part
        score = score - part.double()
    C, LSE = c.run(workspace)
    _check_few(c, C, few)
    c.check(C, LSE)


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("news,lengths,q,kv,d,group,few", MIXES)
def test_few_rows_of_any_values(news, lengths, q, kv, d, group, few, workspace, fmt):
    c = Case(news, lengths, q, kv, d, 16, 0, 0, group, fmt, seed=d + q + 1)
    _check_few(c, c.run(workspace)[0], few)
