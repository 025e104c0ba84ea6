"""Tensors with 8-bit states round by random bits of their own (CPU only: nothing is launched)."""
import torch

import paper_2408_09697_amd as heta


def seeds_of(head):
    head.grads = {"W": torch.zeros_like(head.W), "bias": None}
    return [item[5] for item in head.adamw_items() if len(item) > 5]


def test_heads_that_are_given_no_seed_have_one_of_their_own():
    W = torch.zeros(4, 8)
    heads = [heta.ClassifierHead(None, W, state_bits=8) for _ in range(5)]
    seeds = [s for h in heads for s in seeds_of(h)]
    assert len(seeds) == 5 and len({s & 0xffffffff for s in seeds}) == 5
    # a trainer's count its tensors from its seed on, 0 unless told otherwise
    assert all((s & 0xffffffff) >= 1 << 31 for s in seeds)
    assert [s for h in heads for s in seeds_of(h)] == seeds
    assert seeds_of(heta.ClassifierHead(None, W, state_bits=8, seed=0)) == [0]
    assert seeds_of(heta.ClassifierHead(None, W, state_bits=8, seed=5)) == [5]
