"""Latent attention into outputs anywhere on a 16-byte boundary: results are written in pieces of 32 bytes, which such an address need not
be a multiple of."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2512_23367_b200 as pq
from test_gpu_expanded import Call as Expanded
from test_gpu_latent import Call as Absorbed

pytestmark = pytest.mark.gpu


def _shifted(call, halves):
    """The call's output again, `halves` FP16 values behind a 32-byte boundary, with what lies around it."""
    n = call.out.numel()
    room = torch.full((n + 64,), 7.0, dtype=torch.float16, device=call.out.device)
    assert room.data_ptr() % 32 == 0
    call.out = room[halves: halves + n].view(call.out.shape)
    assert call.out.data_ptr() % 32 == 2 * halves % 32
    return room


def _check(call, rows):
    good = call().clone()
    for halves in (8, 24, 16):
        room = _shifted(call, halves)
        got = call()
        assert pq.pq_device_status() == 0
        assert torch.equal(got[:rows], good[:rows]) and (got[rows:] == 7).all()
        assert (room[:halves] == 7).all() and (room[halves + got.numel():] == 7).all()


# units as a whole, in two or three parts, in many parts (which are joined by more threads)
ABSORBED = {"whole": (16, [1, 2], [130, 70], 16), "parts": (128, [1, 1, 2, 1], [1500, 700, 1290, 2000], 64), "many_parts": (16, [1], [9000], 64)}
EXPANDED = {"whole": (3, [80, 1, 129], [80, 1, 300]), "parts": (2, [100, 300, 5], [500, 1340, 1000]), "many_parts": (2, [2], [9000])}


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("kind", list(ABSORBED))
def test_absorbed_form(kind, workspace, latent):
    heads, new, total, page = ABSORBED[kind]
    _check(Absorbed(ref.latent_inputs(heads, latent, page, new, total, seed=1, gap=2), 0.04, workspace), sum(new))


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("kind", list(EXPANDED))
def test_expanded_form(kind, workspace):
    heads, new, total = EXPANDED[kind]
    _check(Expanded(ref.expanded_inputs(heads, new, total, seed=1, gap=2), 192 ** -0.5, workspace), sum(new))


def test_a_slice_of_a_wider_allocation_holds_the_formula():
    heads, new, total, page = ABSORBED["parts"]
    d = ref.latent_inputs(heads, 512, page, new, total, seed=2)
    call = Absorbed(d, 0.04)
    _shifted(call, 8)
    y, bound = ref.latent_attention(d, 0.04)
    assert (np.abs(call().cpu().numpy().astype(np.float64) - y) <= bound).all() and pq.pq_device_status() == 0


@pytest.mark.parametrize("kind", ["whole", "parts"])
def test_operands_that_begin_at_one_address(kind):
    """Queries, keys and values as columns of one matrix, from its first one on."""
    heads, new, _ = EXPANDED[kind]
    d = ref.expanded_inputs(heads, new, new, seed=5)
    d["q"] = d["kv"][:, : heads * 192].copy()
    apart = Expanded(d, 192 ** -0.5)
    want = apart().clone()
    together = Expanded(d, 192 ** -0.5)
    together.q = together.kv.flatten(1)[:, : heads * 192].unflatten(1, (heads, 192))
    assert together.q.data_ptr() == together.kv.data_ptr()
    assert torch.equal(together(), want) and pq.pq_device_status() == 0
