"""relation_sample's launcher takes the number of SMs from the device, as the other serving calls' do."""
import os
import re

import pytest

from paper_2608_20172_gb300 import build as libbuild


@pytest.mark.parametrize("name", ["relation_sample", "relation_plan", "relation_paged"])
def test_sms_are_asked_for(name):
    with open(os.path.join(libbuild.CSRC, name + ".cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert "cudaDevAttrMultiProcessorCount" in code
    assert not re.search(r"\b152\b", code)
