"""GPU: what a prompt's bf16 output is read out from.  Outputs of either type are formed alike and rounded once, so a bf16 output
is the float output of the same call, rounded -- bit for bit, and there is no bound to derive."""
import pytest
import torch

from paper_2609_04098_b200 import binding as nv
from tests import gdn_ref
from tests import gpu_util as gu
from tests.test_gpu_gdn import check_out, dev

pytestmark = pytest.mark.gpu


def both(ins, lens, **kw):
    """(o, state) of one call with float output and one with bf16 output."""
    Hk, Hv = ins[0].shape[1], ins[2].shape[1]
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=gu.DEV)
    pool = 0.3 * torch.randn(len(lens), Hv, 128, 128, generator=torch.Generator().manual_seed(3))
    out = []
    for f32 in (True, False):
        ws = nv.alloc_gdn_workspace(gu.DEV, sum(lens), len(lens), Hk, Hv, f32)
        state = pool.to(gu.DEV)
        out.append((nv.nvfp4_gdn_prefill(*ins, state, cu, ws, out_f32=f32, **kw), state))
        assert nv.device_status(ws) == 0
    return out, pool


# one chunk, several, a range of its own (more than 48 chunks of one sequence), several value heads of a key head per CTA
@pytest.mark.parametrize("lens,Hk,Hv", [([1], 1, 1), ([17], 16, 48), ([64, 65, 1, 130], 2, 4), ([64 * 70 + 5], 1, 3), ([33] * 60, 16, 48)])
@pytest.mark.parametrize("decay_first", [False, True])
def test_bf16_output_is_the_float_output_rounded(lens, Hk, Hv, decay_first):
    ins = dev(gdn_ref.inputs(21, sum(lens), Hk, Hv, l2norm=True))
    ((o32, s32), (o16, s16)), _ = both(ins, lens, l2norm=True, decay_first=decay_first)
    assert torch.equal(s32, s16)
    assert torch.equal(o32.to(torch.bfloat16), o16)


def test_bf16_output_where_the_read_out_cancels():
    # every odd token overwrites, under the same key, a value about a thousand times its own: what is read out is the small
    # difference of q.S and P U.  The bound is the one of float outputs and a rounding; operands of 11 bits would miss it by far.
    T, Hk, Hv = 128, 1, 2
    q, k, v, a, b, A_log, dtb = gdn_ref.inputs(22, T, Hk, Hv, a_log=(1e-4, 2e-4))
    b[:] = 8.0                                             # beta close to 1
    k[1::2] = k[0::2].clone()
    q.copy_(k)
    v[0::2] = (1000.0 * v[0::2].float()).to(torch.bfloat16)
    ins = (q, k, v, a, b, A_log, dtb)
    (_, (o16, _)), pool = both(dev(ins), [T])
    want, _, m = gdn_ref.recurrence(*ins, pool[0])
    check_out(o16, want, m)
