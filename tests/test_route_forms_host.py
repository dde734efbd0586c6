"""The router's kernels that are built are those that a call can reach: the forms that the rule of the sizes gives over all of them, and no other."""
import os
import re

import paper_1610_06209_amd as package

LIBRARY = os.path.join(os.path.dirname(package.__file__), "libspinner.so")


def built(kernel):
    with open(LIBRARY, "rb") as f:
        return {(int(a), int(b)) for a, b in re.findall(rb"[0-9]" + kernel + rb"I[^E]*?Li([0-9]+)ELi([0-9]+)E", f.read())}


def forms(grad):
    """(lanes a row, experts a lane) by the rule: four lanes for many rows of up to 64 experts, 64 for few rows, 16 otherwise where they hold a row."""
    found = set()
    for count in range(1, 1025):
        for groups in [1] if grad else [g for g in range(1, 65) if count % g == 0]:
            log = (groups - 1).bit_length()
            part = {n: -(-(count // groups) // (n >> log)) if n >> log else 1 << 20 for n in (4, 16, 64)}
            for rows in (1, 2049, 1 << 20):
                for few_choices in (True, False):                   # up to eight, which four lanes hold
                    if rows == 1 and not grad and part[64] <= 4:
                        found.add((64, 1 if part[64] <= 1 else 4))
                    elif rows > 32768 and few_choices and part[4] <= 16:
                        found.add((4, 8 if part[4] <= 8 else 16))
                    elif part[16] <= 16:
                        found.add((16, next(r for r in (1, 4, 8, 16) if part[16] <= r)))
                    else:
                        found.add((64, next(r for r in (8, 16, 32) if part[64] <= r)))
    return found


def test_forms_that_are_built_are_reached():
    assert built(b"route_kernel") == forms(False)
    assert built(b"route_grad_kernel") == forms(True)
