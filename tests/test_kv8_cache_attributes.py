"""A Kv8Cache says what the calls that take it read, also after its attributes are set; nothing is launched, so no GPU is needed."""
import copy

import pytest
import torch

import paper_2605_15609_amd as psd
from paper_2605_15609_amd import binding as B


def cache(**kw):
    return psd.Kv8Cache.empty(2, 3, 64, 20000, device="cpu", **kw)


def test_the_length_that_is_set_is_the_length_that_calls_see():
    c = cache()
    q = torch.zeros((2, 1, 6, 64), dtype=torch.bfloat16)
    assert (c.length, c.c.len) == (20000, 20000)
    plan = B.attention_kv8_plan(q, c)
    c.length = 64
    assert (c.length, c.c.len) == (64, 64) and B.attention_kv8_plan(q, c)[2] < plan[2]
    c.length = c.capacity
    assert B.attention_kv8_plan(q, c) == plan
    for bad in (-1, c.capacity + 1):
        with pytest.raises(psd.PsdError):
            c.length = bad
    assert (c.length, c.c.len) == (c.capacity, c.capacity)


def test_lens_that_are_set_are_the_lens_that_calls_read():
    first, second = torch.ones(2, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    c = cache(lens=first)
    assert c.c.lens == first.data_ptr()
    c.lens = second
    assert c.lens is second and c.c.lens == second.data_ptr()
    for bad in (torch.ones(3, dtype=torch.int32), torch.ones(2), torch.ones(4, dtype=torch.int32)[::2], torch.ones(2, dtype=torch.int32, device="meta")):
        with pytest.raises(psd.PsdError):
            c.lens = bad
    assert c.lens is second and c.c.lens == second.data_ptr()
    c.lens = None
    assert c.lens is None and c.c.lens is None


def test_the_sequences_of_a_unit_that_are_set_are_checked_anew():
    c = cache()
    q = torch.zeros((2, 4, 6, 64), dtype=torch.bfloat16)
    assert B.attention_kv8_plan(q, c)[1] > 0
    c.seqs_per_unit = 2
    assert c.c.seqs_per_unit == 2
    with pytest.raises(psd.PsdError):
        B.attention_kv8_plan(q, c)
    assert B.attention_kv8_plan(torch.zeros((4, 4, 6, 64), dtype=torch.bfloat16), c)[1] > 0
    with pytest.raises(psd.PsdError):
        c.seqs_per_unit = 1 << 40


@pytest.mark.parametrize("name", ["codes", "scales", "format", "device", "units", "n_kv_heads", "d_head", "capacity", "block", "c", "shapes"])
def test_what_a_cache_was_made_with_stays(name):
    c = cache()
    with pytest.raises(psd.PsdError):
        setattr(c, name, getattr(c, name))


def test_a_copy_has_a_length_and_sequences_of_its_own():
    lens = torch.ones(2, dtype=torch.int32)
    one = cache(lens=lens)
    q = torch.zeros((2, 4, 6, 64), dtype=torch.bfloat16)
    other = copy.copy(one)
    other.length, other.lens, other.seqs_per_unit = 64, None, 2
    assert (one.length, one.c.len, one.c.lens, one.c.seqs_per_unit) == (20000, 20000, lens.data_ptr(), 1) and (other.c.len, other.c.lens, other.c.seqs_per_unit) == (64, None, 2)
    assert B.attention_kv8_plan(q, one)[1] > 0
    with pytest.raises(psd.PsdError):
        B.attention_kv8_plan(q, other)
