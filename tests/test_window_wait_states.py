"""The wait states of test_wait_states.py in the emitted code of the windowed-attention kernels, which write their copies and some matrix
instructions as inline assembly too."""
import pytest
import test_wait_states as waits

emitted = waits.emitted
FILES = ("window_fwd.hip", "window_bwd.hip")


@pytest.mark.parametrize("source", FILES)
def test_wait_states_of_the_emitted_code(source, emitted):
    seen = 0
    for name, code in waits.kernels(emitted[source]):
        seen += sum(i.copy for i in code)
        found = waits.faults(code)
        assert not found, f"{name}: {len(found)}, the first: {found[0]}"
    assert seen


@pytest.mark.parametrize("source", FILES)
def test_transcendental_results_have_a_wait_state(source, emitted):
    for name, code in waits.kernels(emitted[source]):
        found = waits.transcendental_results_used_at_once(code)
        assert not found, f"{name}: {len(found)}, the first: {found[0]}"
