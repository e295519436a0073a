"""Registers that the chunk kernels keep in scratch memory, form by form.  Their launch bounds hold the count at 168 or 256 whatever the code needs: what it
needs more shows here alone.  No GPU needed."""
import re

import pytest

from tests.test_chunk_resources import kernels  # noqa: F401 (a fixture)

# looked up once a tile or a group of rows (own positions, intervals, addresses): attention 1 appending, 5 shaped, 6 with a bias as well; scores 2
KNOWN = {r"chunk_attend_kernelILi128ELb0ELb0ELb1EE": 1, r"chunk_attend_kernelILi128ELb1ELb0ELb0EE": 5, r"chunk_attend_kernelILi128ELb1ELb1ELb0EE": 6,
         r"chunk_scores_kernelILi128ELb1ELb0EE": 2}


def test_no_more_registers_in_scratch_memory_than_known(kernels):  # noqa: F811
    found = {n: k for n, k in kernels.items() if re.search(r"5dynts\d+(chunk|rotate)_", n)}
    assert len(found) >= 8 + 4 + 6 + 6 + 2
    for name, k in found.items():
        known = [most for form, most in KNOWN.items() if re.search(form, name)]
        assert k["vgpr_spill_count"] <= (known[0] if known else 0), name


@pytest.mark.parametrize("form", sorted(KNOWN))
def test_the_known_forms_are_there(kernels, form):  # noqa: F811
    assert sum(1 for n in kernels if re.search(form, n)) == 1
