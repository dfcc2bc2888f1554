"""Alternatives of short rows and short parts, on both sides of where a part is spread over all of its CTA's warps."""
import pytest
import torch

from helpers import dev, umim
from test_gpu_logprobs import check_forward, forward, logits

pytestmark = pytest.mark.gpu

# a warp takes 2048 (fp32: 1024) elements side by side, a CTA 16384 (8192); 32 groups to a busy warp, 2 / 3 of them alternatives
SHAPES = [(2048, 21), (2048, 22), (2049, 42), (2049, 43), (4097, 64), (4097, 65), (8192, 85), (8192, 86), (8193, 1), (8193, 85),
          (100, 21), (31, 22), (16383, 20)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,n_top", SHAPES)
def test_short_rows(dtype, V, n_top):
    m, dv = umim(), dev()
    R = 620 if V < 8192 else 330
    V = V if dtype != "fp32" else (V + 1) // 2
    x = logits(V + n_top, R, V, dtype)
    x[1, :V] = x[1, :1]                     # one value everywhere
    x[2, :V] = -float("inf")
    x[2, V // 2:V // 2 + 3] = 1.0           # three allowed
    x[3, :V] = torch.finfo(x.dtype).min
    x[3, V - 2:V] = 2.0                     # masked by the lowest value
    x[4, :V] = x[4, :V].sort(descending=True)[0]
    x[5, :V] = x[5, :V].sort()[0]
    out = forward(m, x, dv, V, None, 1.0, n_top)
    ids = x[:, :V].float().sort(dim=1, descending=True, stable=True)[1][:, :n_top]
    gone = torch.gather(x[:, :V].float(), 1, ids) == -float("inf")
    want = torch.full((R, n_top), -1, dtype=torch.int64)
    want[:, :ids.shape[1]] = ids.masked_fill(gone, -1)
    assert torch.equal(out["top_ids"].cpu().long(), want)
    pick = [0, 1, 2, 3, 4, 5, 151, 152, R - 1]
    check_forward({k: (v[pick] if v is not None else None) for k, v in out.items()}, x[pick], V, None, 1.0, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [32000, 20003])
@pytest.mark.parametrize("R", [1, 16, 64, 100])
@pytest.mark.parametrize("n_top", [5, 21, 43, 64, 86, 128])
def test_short_parts_of_divided_rows(dtype, V, R, n_top):
    m, dv = umim(), dev()
    x = logits(V + R + n_top, R, V, dtype)
    out = forward(m, x, dv, V, None, 1.0, n_top)
    ids = x[:, :V].float().sort(dim=1, descending=True, stable=True)[1][:, :n_top]
    assert torch.equal(out["top_ids"].cpu().long(), ids)
