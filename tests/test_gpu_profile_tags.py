"""Launches of the step in a profile (chgnet_profile_start)."""
import numpy as np
import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw,tag", [({}, "k_embed_bwd_Z"), (dict(conservative=True), "kd_embed")])
@pytest.mark.parametrize("copies", [2, 8, 16])
def test_profile_keeps_the_element_tables_tag(copies, kw, tag):
    """2,158, 8,632 and 17,264 atoms: the table's gradient in one kernel, in the operator's one launch and in its ordering."""
    b = synth.make_batch("triclinic40")
    b = synth.Batch(np.concatenate([[0]] + [b.atom_ptr[1:] + i * b.n_atoms for i in range(copies)]).astype(np.int32),
                    np.tile(b.pos, (copies, 1)), np.tile(b.lattice, (copies, 1, 1)), np.tile(b.Z, copies))
    hp = bd.hparams(d=64, n_layers=1, **kw)
    p = torch.as_tensor(synth.make_params(64, 1)).cuda()
    targets = [torch.as_tensor(x).cuda() for x in synth.make_targets(b)]
    db, g, ws = bd.DeviceBatch.from_host(b), bd.DeviceGraph(b.n_atoms, 64, 16, 64), bd.Workspace()
    bd.step(hp, db, g, p, targets, ws)
    bd.profile_start(10000)
    try:
        bd.step(hp, db, g, p, targets, ws)
        torch.cuda.synchronize()
    finally:
        tags = bd.profile_stop()
    assert tag in tags and not [t for t in tags if t.startswith(("k_embed_count", "k_embed_place", "k_embed_runs", "k_embed_join", "k_embed_few"))]
