"""Scales of 8-bit floats as views (``paper_1803_03288_amd.layers.Float8``): one row of scales for all rows, rows apart, rows that share bytes; the same bits as scales that lie by themselves."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_update import L  # noqa: F401


def bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("rows,cols", [(3, 100), (70, 600), (300, 1025)])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scales_as_views(L, rows, cols, block, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.rand(rows, cols, generator=g, device="cuda") + 1.01) * 0.49      # all blocks have one scale (0.49 to 0.99; the largest above 0.875)
    x[:, ::50] = x[:, -1] = 0.98                            # (a last block of one column too)
    dy = torch.randn(rows, 70, generator=g, device="cuda").to(dtype)
    w = L.quantize_f8(torch.randn(70, cols, generator=g, device="cuda"), 128)
    r = L.quantize_f8(x, block)
    up, along = r.scale.shape
    plain = r.scale.view(torch.uint8)[:, :-(-cols // 128)]
    assert torch.equal(plain, plain[:1].expand_as(plain))
    room = torch.zeros(up * along + along, dtype=torch.uint8, device="cuda")
    room[:] = plain[0, 0]
    wide = torch.zeros(up, along + 8, dtype=torch.uint8, device="cuda")
    wide[:, 4:4 + along] = r.scale.view(torch.uint8)
    views = [r.scale.view(torch.uint8)[:1].expand(up, along), room[:1].expand(up, along), room.as_strided((up, along), (1, 1)), wide[:, 4:4 + along], wide[:, 4:4 + plain.shape[1]]]
    want = (L.dequantize_f8(r, dtype), L.linear_f8(r, w, dtype=dtype), *L.linear_f8_backward(dy, r, w))
    for v in views:
        s = L.Float8(r.q, v.view(torch.float8_e8m0fnu), cols, block)
        got = (L.dequantize_f8(s, dtype), L.linear_f8(s, w, dtype=dtype), *L.linear_f8_backward(dy, s, w))
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want))
