"""What the operators around the attention rest on that no run can show, and sizes at the ends of what they take.  No GPU needed."""
import os
import re

import pytest

from paper_2605_11354_b200 import binding as lt
from paper_2605_11354_b200 import build as lb


@pytest.fixture(scope="module", autouse=True)
def library():
    lb.build()
    return lt.lib()


def test_arrivals_at_another_cta_have_its_scope():
    """An arrival on a barrier of another CTA orders nothing for the thread that waits there unless its scope is the cluster (or
    it orders nothing on purpose); without a scope it is the CTA's."""
    found = []
    for name in sorted(os.listdir(lb.CSRC)):
        with open(os.path.join(lb.CSRC, name)) as f:
            found += [(name, op) for op in re.findall(r"mbarrier\.arrive[\w.:]*", f.read()) if "shared::cluster" in op]
    assert found and all(".cluster." in op.replace("shared::cluster", "") for _, op in found), found
