"""Lists of gradients in which something is written where something else is read, or written twice: one CTA would write what
another reads, in no order."""
import random

import pytest
import torch

from paper_2609_32197_b200 import binding
from test_layer_host import INVALID, refused
from test_step_host import grads, table_of


def test_an_output_in_the_place_of_another_gradient():
    for bad in (grads((4096, 8), (8192, 8), outs=[8192, 65536]),  # where the second is read
                grads((4096, 8), (8192, 8), outs=[65536, 4096]),
                grads((4096, 8), (8192, 8), outs=[8192, 4096]),  # exchanged
                grads((4096, 8), (8192, 8), outs=[8206, 65536]),  # its last value
                grads((4096, 8), (8192, 8), outs=[8178, 65536]),  # ... and its first
                grads((4096, 8), (8192, 8), outs=[8192, 8192]),
                grads((4096, 800), (4104, 8), outs=[4096, 65536]),  # in place, around another
                grads((4096, 8), outs=[4098]), grads((4096, 8), outs=[4082])):  # beside its own place
        refused(INVALID, binding.sparsp_grad_table, bad, table_of(bad))
    a, b, o = torch.zeros(4), torch.zeros(6), torch.zeros(4)
    with pytest.raises(binding.SparspError):
        binding.make_grad_list([a, o], [o, torch.zeros(4)])
    binding.make_grad_list([a, b], [o, b])


def test_what_does_not_meet_is_taken():
    for good in (grads((4096, 8), (8192, 8), outs=[4096, 8192]),  # all in place
                 grads((4096, 8), (8192, 8), outs=[65536, 8192]),  # some
                 grads((4096, 8), (4096, 8), outs=[8192, 65536]),  # one gradient twice, to two places
                 grads((4096, 8), (4100, 8), outs=[65536, 8192]),
                 grads((4096, 8), (4112, 8), outs=[4080, 4128]),  # one behind the other
                 grads((8192, 8), (4096, 0), outs=[4096, 8192]),  # nothing at the other place
                 grads((8192, 8), (4096, 8), outs=[8192, 65536])):
        binding.sparsp_grad_table(good, table_of(good))


def test_against_every_pair():
    rng = random.Random(5)
    seen = set()
    for _ in range(3000):
        n = rng.randint(1, 5)
        places = [1024 + 2 * rng.randint(0, 60) for _ in range(2 * n)]
        sizes = [rng.choice((0, 1, 3, 8, 20)) for _ in range(n)]
        outs = [places[i] if rng.random() < 0.3 else places[n + i] for i in range(n)]

        def meet(a, na, b, nb):
            return na > 0 and nb > 0 and a < b + 2 * nb and b < a + 2 * na

        bad = any(meet(outs[i], sizes[i], places[j], sizes[j]) and not (i == j and outs[i] == places[j]) or
                  i != j and meet(outs[i], sizes[i], outs[j], sizes[j]) for i in range(n) for j in range(n))
        lst = grads(*zip(places, sizes), outs=outs)
        seen.add(bad)
        if bad:
            refused(INVALID, binding.sparsp_grad_table, lst, table_of(lst))
        else:
            binding.sparsp_grad_table(lst, table_of(lst))
    assert seen == {False, True}
