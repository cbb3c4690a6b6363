"""A preset's schedule refuses drafted tokens, before anything is launched."""
import pytest

from paper_2601_18383_b200 import presets


@pytest.mark.parametrize("options", [dict(stage=True), dict(tree=object()), dict(stage=True, tree=object(), sinks=2)])
def test_drafted_tokens_are_refused(options):
    run = object.__new__(presets.PresetRun)  # (no cache: nothing of it may be touched)
    with pytest.raises(ValueError, match="room behind its budget"):
        run.extend(None, None, None, None, **options)
