"""One token's residual stream updated in place inside a wider buffer: a single row has no stride to speak of, so the residual is
Y itself whatever the two strides say."""
import pytest
import torch

from paper_2609_04098_b200 import binding as nv
from tests import gpu_util as gu
from tests.test_epilogue_abi import L, P, _bf16, _codes, _epi  # noqa: F401 (L is the fixture)


@pytest.mark.parametrize("call", [_codes, _bf16])
def test_strides_of_one_row_do_not_matter(L, call):  # noqa: F811
    assert call(L, _epi(residual=P, ldr=16), M=1, ldy=40, ws=None) == 5          # as far as the next check (no workspace)
    assert call(L, _epi(residual=P, ldr=40), M=1, ldy=16, ws=None) == 5
    assert call(L, _epi(residual=P, ldr=16), M=2, ldy=40, ws=None) == 2          # two rows: they do
    assert call(L, _epi(residual=P + 2, ldr=16), M=1, ldy=40, ws=None) == 2      # and a shifted row still overlaps
    assert call(L, _epi(residual=P + 32, ldr=16), M=1, ldy=40, ws=None) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2])
@pytest.mark.parametrize("bf16_in", [False, True])
@pytest.mark.parametrize("out_f32", [False, True])
def test_columns_of_a_wider_buffer_updated_in_place(M, bf16_in, out_f32):
    from tests.test_gpu_epilogue import Layer, extras
    N, dt = 520, torch.float32 if out_f32 else torch.bfloat16
    layer = Layer(15, M, N, 512)
    _, r = extras(3, M, N, dt, bias=False)
    want = layer.run(bf16_in, residual=r, out_f32=out_f32)
    wide = torch.full((M, 2 * N + 24), 9.0, dtype=dt, device=gu.DEV)
    y = wide[:, 8:8 + N]
    y.copy_(r)
    layer.run(bf16_in, residual=y, out=y)
    assert torch.equal(y, want)
    assert (wide[:, :8] == 9).all() and (wide[:, 8 + N:] == 9).all()
    assert nv.device_status(layer.ws) == 0
