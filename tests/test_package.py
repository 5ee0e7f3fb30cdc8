"""The package offers the decoding calls under its own name."""

import pytest

package = pytest.importorskip("paper_2408_03675_amd")


@pytest.mark.parametrize("name", [
    "Step", "Rotation", "Prefix", "rotate_append", "prefix_workspace", "prefix_attention", "sample_workspace", "sample",
    "Pages", "pages_assign", "paged_append", "paged_workspace", "paged_attention", "beam_workspace", "beam_select",
    "beam_reorder",
])
def test_decoding_calls_are_the_package_s(name):
    assert getattr(package, name) is getattr(package.nacl, name)
