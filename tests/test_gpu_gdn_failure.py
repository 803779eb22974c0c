"""GPU: the prefill whose waits run out.  Nothing hangs or faults: its second kernel starts under the tail of the first and waits
for it, and with a limit of 1 ns that wait gives up, the call ends and its status says so."""
import pytest
import torch

from paper_2609_04098_b200 import binding as nv
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out_f32", [False, True])
def test_prefill_that_gives_up_leaves_whole_states(out_f32):
    # 64 value heads on one key head make long CTAs of the preparation, four of which share an SM; 48 chunks more than fit at
    # once leave most SMs to the second kernel while those run
    sms = torch.cuda.get_device_properties(gu.DEV).multi_processor_count
    Hk, Hv, n = 1, 64, 8
    lens = [64 * ((4 * sms + 48) // n)] * n
    T = sum(lens)
    gen = torch.Generator(device=gu.DEV).manual_seed(31)

    def r(*shape):
        return torch.randn(*shape, generator=gen, device=gu.DEV)
    bf16 = torch.bfloat16
    ins = (r(T, Hk, 128).to(bf16), r(T, Hk, 128).to(bf16), r(T, Hv, 128).to(bf16), r(T, Hv).to(bf16), r(T, Hv).to(bf16),
           torch.full((Hv,), -2.0, device=gu.DEV), 0.1 * r(Hv))
    cu = torch.tensor([sum(lens[:i]) for i in range(n + 1)], dtype=torch.int32, device=gu.DEV)
    pool = 0.3 * r(n, Hv, 128, 128)
    ws = nv.alloc_gdn_workspace(gu.DEV, T, n, Hk, Hv, out_f32)

    def go():
        state = pool.clone()
        out = torch.full((T, Hv, 128), 7.0, dtype=torch.float32 if out_f32 else bf16, device=gu.DEV)
        nv.nvfp4_gdn_prefill(*ins, state, cu, ws, l2norm=True, out=out)
        return state, out
    state, out = go()
    assert nv.device_status(ws) == 0
    torch.cuda.synchronize()
    try:
        nv.set_wait_limit_ns(1)
        cut, cut_out = go()
        assert nv.device_status(ws) == 8                       # NVFP4_ERR_TIMEOUT
    finally:
        nv.set_wait_limit_ns(0)
    old, new = ((cut == x).flatten(2).all(-1) for x in (pool, state))
    assert (old | new).all() and old.any()
    rows = cut_out.view(n, -1, Hv, 128)
    done = new[:, None, :, None].expand_as(rows)
    assert torch.equal(rows[done], out.view(n, -1, Hv, 128)[done])
    nv.workspace_reset(ws)
    again, again_out = go()
    assert nv.device_status(ws) == 0 and torch.equal(again, state) and torch.equal(again_out, out)
