"""GPU: keys and queries far below the epsilon of the length they are divided by, x / sqrt(sum x^2 + 1e-6).  A power-of-two scale
cancels out of every step, so the bounds are those of ordinary keys (test_gpu_gdn)."""
import pytest
import torch

from paper_2609_04098_b200 import binding as nv
from tests import gdn_ref
from tests import gpu_util as gu
from tests.test_gpu_gdn import check_out, check_state, dev

pytestmark = pytest.mark.gpu


def inputs(e_k, e_q, T=70):
    ins = list(gdn_ref.inputs(23, T, 1, 2, l2norm=True))
    ins[0] = (ins[0].float() * 2.0 ** e_q).to(torch.bfloat16)
    ins[1] = (ins[1].float() * 2.0 ** e_k).to(torch.bfloat16)
    return ins


# either side of where the kernel's scale makes the sum of squares negligible (rows around 2^-37), of where the scale squared
# leaves binary32 (2^-64), and the smallest normal numbers
@pytest.mark.parametrize("e", [-12, -36, -37, -38, -39, -40, -63, -66, -100, -120])
def test_prefill_of_tiny_keys_and_queries(e):
    T = 70
    cu = torch.tensor([0, T], dtype=torch.int32, device=gu.DEV)
    ws = nv.alloc_gdn_workspace(gu.DEV, T, 1, 1, 2, True)
    for e_k, e_q in ((e, 0), (0, max(e, -100))):            # (outputs below 2^-126 would have fewer bits)
        ins = inputs(e_k, e_q)
        state = torch.zeros(1, 2, 128, 128, device=gu.DEV)
        o = nv.nvfp4_gdn_prefill(*dev(ins), state, cu, ws, l2norm=True, out_f32=True)
        want, S, m = gdn_ref.recurrence(*ins, torch.zeros(2, 128, 128), l2norm=True)
        check_state(state[0], S)
        check_out(o, want, m)


@pytest.mark.parametrize("e", [-40, -66, -100])
def test_prompt_and_tokens_agree_on_tiny_keys(e):
    T = 3
    ins = inputs(e, 0, T)
    d = dev(ins)
    state, step = (torch.zeros(1, 2, 128, 128, device=gu.DEV) for _ in range(2))
    cu = torch.tensor([0, T], dtype=torch.int32, device=gu.DEV)
    ws = nv.alloc_gdn_workspace(gu.DEV, T, 1, 1, 2, True)
    nv.nvfp4_gdn_prefill(*d, state, cu, ws, l2norm=True, out_f32=True)
    for t in range(T):
        nv.nvfp4_gdn_decode(*[x[t:t + 1] for x in d[:5]], *d[5:], step, l2norm=True, out_f32=True)
    _, S, _ = gdn_ref.recurrence(*ins, torch.zeros(2, 128, 128), l2norm=True)
    check_state(state[0], S)
    check_state(step[0], S)
