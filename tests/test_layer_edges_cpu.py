"""What the operators around the attention rest on that no run can show, and sizes at the ends of what they take.  No GPU needed."""
import os
import re

import numpy as np
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


def test_the_workspace_has_room_on_every_device():
    """The rule that cuts the rows depends on the number of SMs; what the size query asks for has to do on all of them (a part of a
    GPU has a few, a later one may have more)."""
    g = np.random.default_rng(0)
    sizes = [(10992, 1024, 1024), (10992, 1024, 4096), (777, 1184, 1000), (1, 32, 8), (512, 32, 8), (40000, 64, 64), (43968, 4096, 1024)]
    sizes += [(int(2 ** g.uniform(0, 17)), 32 * int(2 ** g.uniform(0, 8)), int(2 ** g.uniform(0, 13))) for _ in range(60)]
    cut = 0
    for rows, d_in, d_out in sizes:
        room = lt.lite3r_linear_mx_workspace(rows, d_in, d_out)
        for sms in (1, 2, 3, *range(8, 300, 4)):
            parts, size = lt.lite3r_linear_mx_parts(rows, d_in, d_out, sms)
            steps = -(-rows // 64)
            assert 1 <= parts <= 16 and (parts - 1) * -(-steps // parts) < steps, (rows, d_in, d_out, sms, parts)  # none is empty
            assert size <= room, (rows, d_in, d_out, sms, parts)
            cut += parts > 1
    assert cut > 100


@pytest.mark.parametrize("args", [(0, 32, 8, 148), (5, 0, 8, 148), (5, 32, 0, 148), (5, 32, 8, 0), (5, 48, 8, 148)])
def test_parts_refuse_what_is_no_layer(args):
    with pytest.raises(lt.Lite3rError):
        lt.lite3r_linear_mx_parts(*args)


def test_waits_for_another_cta_have_its_scope():
    """A kernel that sends arrivals to its pair's first CTA waits for them there at cluster scope, too."""
    for name in sorted(os.listdir(lb.CSRC)):
        with open(os.path.join(lb.CSRC, name)) as f:
            text = f.read()
        if not name.endswith(".cu") or "mbar_arrive_cluster" not in text:
            continue
        waits = re.findall(r"(mbar_wait_cluster_clearing(?:<true>)?\(\s*|wait_read\(\s*|mbar_wait_clearing\(\s*)&bars->(acc_empty|shared_read)", text)
        assert any(how.startswith(("mbar_wait_cluster", "wait_read")) for how, _ in waits), (name, waits)
