"""Rows read out of a 4-bit cache into interleaved planes of one buffer, on the GPU."""
import pytest
import torch

from kv4_reference import stored
from paper_2412_05693_amd import batchmax as bmx
from test_gpu_kv4 import gen, make, rows

pytestmark = pytest.mark.gpu


def test_both_planes_in_one_buffer():
    """k in rows 0..3 and v in rows 4..7 of every unit of one tensor: no row twice."""
    b, hk, d, n = 2, 3, 64, 4
    att = make(b=b, heads=hk, kv_heads=hk, d=d)
    g = gen(5)
    k, v = rows(g, (b, hk, n, d), "bf16"), rows(g, (b, hk, n, d), "bf16")
    att.write_rows(3, k, v)
    out = torch.full((b, hk, 2 * n, d), 7.0, dtype=torch.bfloat16, device="cuda")
    bmx.bm_kv4_read(att.dims, att.cache, 3, n, out.data_ptr(), out.data_ptr() + n * d * 2, 2 * n,
                    torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out[:, :, :n].cpu().double(), stored(k))
    assert torch.equal(out[:, :, n:].cpu().double(), stored(v))
