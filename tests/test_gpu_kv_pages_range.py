"""The ends of the 8-bit pages' range, on a real MI355X: what ntp_qk_norm_append_shard stores of bf16's largest numbers, and that ntp_attn_chunk_shard reads finite values back as such.

A sequence of one token has a weight of exactly 1, so that its output is its value: the e4m3 number times the power of two, which bf16 holds."""
import numpy as np
import pytest

from oracle import block_oracle as B
from tests.test_gpu_attn_chunk import _say, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [1, 40])  # few rows, row tiles
@pytest.mark.parametrize("d", [64, 128])
def test_finite_values_are_read_back_finite(d, group):
    import torch
    import paper_2504_06095_amd as N
    _say(f"8-bit pages of bf16's largest values, heads of {d}, {group} query heads")
    tops = [2.0 ** 127 * f for f in (1.0, 1.75, 1.7578125, 1.875, 1.9296875, 1.9375, 1.9453125, 1.9921875)] + [2.0 ** -111, 448 * 2.0 ** -111, 2.0 ** -126]
    n, page = len(tops), 16
    QKV = torch.zeros(n, (group + 2) * d, dtype=torch.bfloat16, device="cuda")
    V = QKV[:, (group + 1) * d:]
    V[:, 0] = torch.tensor(tops, dtype=torch.float64).to(torch.bfloat16)
    V[:, 1] = -V[:, 0]
    V[:, 2:] = V[:, :1] * torch.linspace(-1, 1, d - 2, device="cuda")
    plan = dict(q_cnt=group, kv_cnt=1, q_off=0, kv_off=0, head_dim=d)
    K8, V8 = (torch.zeros(n, 1, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    Ke, Ve = (torch.zeros(n, 1, page, dtype=torch.uint8, device="cuda") for _ in range(2))
    pages = N.kv_pages(K8, V8, Ke, Ve)
    N.ntp_qk_norm_append_shard(N.kv_append_shape(n, plan, 0), None, pages, QKV, None, torch.arange(n, device="cuda") * page, None)
    table = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    C = torch.empty(n, group * d, dtype=torch.bfloat16, device="cuda")
    N.ntp_attn_chunk_shard(N.attn_chunk_shape(n, n, 1, 1, plan, group), pages, torch.zeros_like(C), None, table, torch.ones(n, dtype=torch.int32, device="cuda"), C)
    torch.cuda.synchronize()
    num, code = B.heads_to_8_bits(f64(V))
    assert np.array_equal(Ve[:, 0, 0].cpu().numpy(), code) and np.array_equal(f64(V8)[:, 0, 0], num)
    back = np.ldexp(num, (code - 127).astype(int)[:, None])
    assert np.abs(back).max() == 1.875 * 2.0 ** 127
    # normal numbers of bf16: exactly; below them half a step of its smallest
    got = f64(C).reshape(n, group, d)
    assert (np.abs(got - back[:, None]) <= np.where(np.abs(back[:, None]) >= 2.0 ** -126, 0.0, 2.0 ** -134)).all()


def test_what_is_not_finite_beside_the_largest_values():
    import torch
    import paper_2504_06095_amd as N
    d, page = 64, 16
    QKV = torch.zeros(1, 2 * d, dtype=torch.bfloat16, device="cuda")
    QKV[0, :4] = torch.tensor([3.38e38, float("inf"), -float("inf"), float("nan")])
    K8, V8 = (torch.zeros(1, 1, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    Ke, Ve = (torch.zeros(1, 1, page, dtype=torch.uint8, device="cuda") for _ in range(2))
    N.ntp_qk_norm_append_shard(N.kv_append_shape(1, dict(q_cnt=0, kv_cnt=1, head_dim=d), 0), None, N.kv_pages(K8, V8, Ke, Ve), QKV, None, torch.zeros(1, dtype=torch.int64, device="cuda"), None)
    k = f64(K8)[0, 0, 0]
    assert k[0] == 240 and np.isnan(k[1:4]).all() and not k[4:].any() and int(Ke[0, 0, 0]) == 247
