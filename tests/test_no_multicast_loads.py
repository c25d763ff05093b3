"""The library runs in processes that use several GPUs (a rank per GPU), where a TMA load with cluster
multicast has no place: no source has one."""
import os
import re

from conftest import ROOT

LOAD = re.compile(r"cp\.async\.bulk[\w.:]*\.multicast")


def test_no_source_has_a_multicast_load():
    assert LOAD.search('"cp.async.bulk.tensor.4d.shared::cluster.global.tile.multicast::cluster"')
    checked = 0
    for folder in ("include", os.path.join("paper_2609_21849_gb300", "csrc")):
        for name in sorted(os.listdir(os.path.join(ROOT, folder))):
            if name.endswith((".cu", ".cuh", ".h")):
                with open(os.path.join(ROOT, folder, name)) as f:
                    joined = re.sub(r'"\s*"', "", f.read())   # (adjacent string literals are one)
                assert not LOAD.search(joined), name
                checked += 1
    assert checked > 20
