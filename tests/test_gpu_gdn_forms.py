"""GPU: the forms of the served recurrence that the sizes of a call choose, each on purpose on its own side of the rule.

  single tokens   a quarter of a head per CTA up to 2 CTAs' worth of heads per SM, a whole head above
  preparation     one value head per CTA; all value heads of a key head once (chunk slots) x (key heads) >= 4 per SM
  prompts         in one piece, or range by range of 32 chunks (one pair of launches each) for few long sequences

Tolerances are those of test_gpu_gdn; where two forms do the same arithmetic in the same order, results are equal bit for bit."""
import pytest
import torch

from paper_2609_04098_b200 import binding as nv
from tests import gdn_ref
from tests import gpu_util as gu
from tests.test_gpu_gdn import check_out, check_state, dev, run_prefill

pytestmark = pytest.mark.gpu


def sms():
    return torch.cuda.get_device_properties(gu.DEV).multi_processor_count


def offsets(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=gu.DEV)


# ------------------------------------------------------------------------------------------ single tokens
@pytest.mark.parametrize("rows,Hk,Hv", [(lambda n: 2 * n // 4, 1, 4), (lambda n: 2 * n // 4 + 1, 1, 4), (lambda n: 37 * n // 148, 16, 32),
                                        (lambda n: 2 * n // 6 + 1, 3, 6)])
@pytest.mark.parametrize("l2norm,decay_first,gates,out_f32", [(True, False, torch.bfloat16, False), (False, True, torch.float32, True)])
def test_decode_on_both_sides_of_the_switch(rows, Hk, Hv, l2norm, decay_first, gates, out_f32):
    B = rows(sms())
    ins = gdn_ref.inputs(B, B, Hk, Hv, gates, l2norm, fused=True)
    gen = torch.Generator().manual_seed(B)
    pool = 0.3 * torch.randn(B + 2, Hv, 128, 128, generator=gen)
    slots = torch.randperm(B + 2, generator=gen)[:B].to(torch.int32)
    slots[1], slots[B - 2] = -1, B + 2                         # padding rows
    state = pool.to(gu.DEV)
    out = torch.full((B, Hv, 128), 7.0, dtype=torch.float32 if out_f32 else torch.bfloat16, device=gu.DEV)
    nv.nvfp4_gdn_decode(*dev(ins), state, slots=slots.to(gu.DEV), l2norm=l2norm, decay_first=decay_first, out=out)
    torch.cuda.synchronize()
    for i in range(B):
        s = int(slots[i])
        if not 0 <= s < B + 2:
            assert (out[i] == 7.0).all()
            continue
        o_ref, S_ref, m = gdn_ref.recurrence(*[t[i:i + 1] for t in ins[:5]], *ins[5:], pool[s], l2norm, decay_first)
        check_out(out[i:i + 1], o_ref, m)
        check_state(state[s], S_ref)
    for s in set(range(B + 2)) - set(slots.tolist()):
        assert torch.equal(state[s].cpu(), pool[s])


def test_decode_forms_agree_on_the_same_rows():
    # the rows of a large batch, alone in calls of one: other lanes hold other columns, so sums may round differently
    B, Hk, Hv = 2 * sms() // 4 + 8, 1, 4
    ins = gdn_ref.inputs(3, B, Hk, Hv, torch.bfloat16, True)
    d = dev(ins)
    pool = (0.3 * torch.randn(B, Hv, 128, 128, generator=torch.Generator().manual_seed(3))).to(gu.DEV)
    together, alone = pool.clone(), pool.clone()
    nv.nvfp4_gdn_decode(*d, together, l2norm=True)
    for i in (0, 1, B // 2, B - 1):
        slot = torch.tensor([i], dtype=torch.int32, device=gu.DEV)
        nv.nvfp4_gdn_decode(*[t[i:i + 1] for t in d[:5]], *d[5:], alone, slots=slot, l2norm=True)
        check_state(alone[i], together[i].cpu())


# ------------------------------------------------------------------------------------------ preparation
def enough(Hk):
    """Sequences whose slots alone make the preparation take every value head of a key head in one CTA."""
    return (4 * sms() + Hk - 1) // Hk


@pytest.mark.parametrize("Hk,Hv", [(2, 6), (4, 8)])
@pytest.mark.parametrize("out_f32,decay_first", [(False, False), (True, True)])
def test_prefill_several_value_heads_per_preparation_cta(Hk, Hv, out_f32, decay_first):
    run_prefill([(i * 5) % 7 for i in range(enough(Hk))], Hk, Hv, seed=Hk, cont=None, l2norm=True, out_f32=out_f32, decay_first=decay_first,
                gates=torch.bfloat16)


@pytest.mark.parametrize("Hk,Hv", [(16, 48), (2, 10)])
@pytest.mark.parametrize("out_f32", [False, True])
def test_prefill_of_many_is_the_prefill_of_each(Hk, Hv, out_f32):
    # the same sequence in a call of its own is prepared one value head at a time
    n = enough(Hk)
    lens = [(i * 37) % 140 for i in range(n)]
    cu = offsets(lens)
    d = dev(gdn_ref.inputs(8, sum(lens), Hk, Hv, torch.bfloat16, True, fused=True))
    pool = torch.randn(n, Hv, 128, 128, generator=torch.Generator(device=gu.DEV).manual_seed(8), device=gu.DEV)
    ws = nv.alloc_gdn_workspace(gu.DEV, sum(lens), n, Hk, Hv, out_f32)
    state = pool.clone()
    o = nv.nvfp4_gdn_prefill(*d, state, cu, ws, l2norm=True, out_f32=out_f32)
    for i in list(range(0, n, max(1, n // 12))) + [n - 1]:
        if lens[i] == 0:
            assert torch.equal(state[i], pool[i])
            continue
        at = slice(int(cu[i]), int(cu[i]) + lens[i])
        S = pool[i:i + 1].clone()
        alone = nv.nvfp4_gdn_prefill(*[t[at] for t in d[:5]], *d[5:], S, offsets([lens[i]]), ws, l2norm=True, out_f32=out_f32)
        assert torch.equal(alone, o[at]) and torch.equal(S[0], state[i])
    assert nv.device_status(ws) == 0


# ------------------------------------------------------------------------------------------ ranges of chunks
def in_ranges(T, nseq, Hv):
    """Pairs of launches that a call should make."""
    chunks = (T + 63) // 64
    assert 2 * nseq * Hv <= sms() and chunks > 48 * nseq, "the sizes of this test no longer make ranges"
    return (chunks + 31) // 32


# a sequence that ends with a range, one token in front of and behind it, others that end earlier, empty ones (the mixed
# has_state of run_prefill: even ones start from zero, odd ones continue), a padding sequence
@pytest.mark.parametrize("lens,slots", [([64 * 64], None), ([64 * 64 - 1], None), ([64 * 64 + 1], None), ([64 * 32, 64 * 120], None),
                                        ([64 * 200, 0, 0, 1], None), ([0, 64 * 128, 64 * 32], [4, 0, -1])])
@pytest.mark.parametrize("out_f32,decay_first", [(False, True), (True, False)])
def test_prefill_in_ranges(lens, slots, out_f32, decay_first):
    Hv = 2
    pairs = in_ranges(sum(lens) + 3, len(lens), Hv)
    before = nv.launch_count()
    run_prefill(lens, 1, Hv, seed=sum(lens), cont=None, l2norm=True, out_f32=out_f32, decay_first=decay_first, slots=slots)
    assert nv.launch_count() - before == 2 * pairs


@pytest.mark.parametrize("out_f32", [False, True])
def test_ranges_are_the_prefill_in_one_piece(out_f32):
    # the model's heads; empty sequences behind the long one bring the average length below what ranges ask for
    T, Hk, Hv = 64 * 70 + 9, 16, min(48, sms() // 2)
    Hk = Hk if Hv % Hk == 0 else 1
    d = dev(gdn_ref.inputs(9, T, Hk, Hv, torch.bfloat16, True, fused=True))
    pool = torch.randn(3, Hv, 128, 128, generator=torch.Generator(device=gu.DEV).manual_seed(9), device=gu.DEV)
    got = []
    for lens in ([T], [T, 0, 0]):
        ws = nv.alloc_gdn_workspace(gu.DEV, T, len(lens), Hk, Hv, out_f32)
        state = pool.clone()
        before = nv.launch_count()
        o = nv.nvfp4_gdn_prefill(*d, state, offsets(lens), ws, l2norm=True, out_f32=out_f32)
        got.append((o, state, nv.launch_count() - before))
        assert nv.device_status(ws) == 0
    assert got[0][2] == 2 * in_ranges(T, 1, Hv) and got[1][2] == 2
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_ranges_replayed_from_a_graph():
    # two prompts' halves and a token behind each other on one workspace, captured: the edges between ranges, calls and forms
    T, Hk, Hv = 64 * 65, 16, min(48, sms() // 2)
    Hk = Hk if Hv % Hk == 0 else 1
    in_ranges(T, 1, Hv)
    d = [t.clone() for t in dev(gdn_ref.inputs(10, T, Hk, Hv, torch.bfloat16, True))]
    state = torch.zeros(1, Hv, 128, 128, device=gu.DEV)
    cu = offsets([T])
    ws = nv.alloc_gdn_workspace(gu.DEV, T, 1, Hk, Hv)
    outs = [torch.empty((T, Hv, 128), dtype=torch.bfloat16, device=gu.DEV) for _ in range(2)]
    tok = torch.empty((1, Hv, 128), dtype=torch.bfloat16, device=gu.DEV)

    def step(sync=lambda: None):
        for o in outs:
            nv.nvfp4_gdn_prefill(*d, state, cu, ws, l2norm=True, out=o)
            sync()
        nv.nvfp4_gdn_decode(*[t[:1] for t in d[:5]], *d[5:], state, l2norm=True, out=tok)
        sync()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in (11, 12):
        for t, x in zip(d, gdn_ref.inputs(seed, T, Hk, Hv, torch.bfloat16, True)):
            t.copy_(x)
        state.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs + [tok, state]]
        state.zero_()
        step(torch.cuda.synchronize)
        assert all(torch.equal(a, b) for a, b in zip(got, outs + [tok, state]))
    assert nv.device_status(ws) == 0
    del graph
