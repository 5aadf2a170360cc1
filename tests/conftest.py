import os
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
for path in (ROOT, HERE):
    if path not in sys.path:
        sys.path.insert(0, path)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


FINISHED = ("a beam that is finished at 12 tokens is held to 140 in its cache, of which 128 are padding that a search behind it would go on from and that takes "
            "the pages of others (tests/test_gpu_beam_loop_ends.py has the same steps with the tokens that the beam has)")

# Tests that hold a wrong value, and which: they run, and are expected to fail there.
WRONG_VALUES = {
    "test_gpu_decoding_loop.py::test_a_prompt_enters_compressed":
        "a prompt behind a shared prefix of 40 tokens is held to positions from 0, where the prefix's own keys stand, and to "
        "weights that leave the prefix out (tests/test_gpu_decoding_loop_state.py has the two as one sequence)",
    "test_gpu_beam_loop.py::test_every_stage_of_many_steps[0-0]": FINISHED,
    "test_gpu_beam_loop.py::test_every_stage_of_many_steps[50-3]": FINISHED,
}


def pytest_collection_modifyitems(items):
    for item in items:
        for name, reason in WRONG_VALUES.items():
            if item.nodeid.endswith(name):
                item.add_marker(pytest.mark.xfail(reason=reason, raises=AssertionError, strict=True))


@pytest.fixture(scope="session")
def gpu():
    """(library binding, device helpers, torch) for the tests marked gpu; the library must be built."""
    import torch
    assert torch.cuda.is_available(), "needs a GPU"
    import paper_2604_18655_amd as lib
    from paper_2604_18655_amd import device
    lib.load_library()
    return lib, device, torch
