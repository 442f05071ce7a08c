"""muon_step in mode 1 at mode 0's exactness where the caller asks for it (MUON_FULL): the update is mode 0's, bit by bit."""
import pytest

from tests.test_muon_plans_cpu import plans  # noqa: F401

# (D, H, L, P, V), other flags: on 256 x 128 tiles without the flag, one short of it, small
MODELS = [((260, 512, 4, 256, 300), 1), ((300, 500, 4, 201, 300), 2), ((64, 128, 2, 256, 3000), 5), ((40, 32, 1, 0, 100), 7)]


def test_the_plan_is_mode_0s(plans):  # noqa: F811
    got = plans(f"""
        out = []
        for dims, flags in {MODELS!r}:
            full, real, half = (plans(model(f, *dims, mode)[0]) for f, mode in ((flags | bl.MUON_FULL, 1), (flags, 0), (flags, 1)))
            out.append([full == real, full[0][3]["exact"] or full[0][3]["tile"] == 3, bad_bytes(dims, flags)])
    """.replace("bad_bytes(dims, flags)", "model(flags | bl.MUON_FULL, *dims, 1)[1] == model(flags, *dims, 0)[1] and wrong(*model(flags | bl.MUON_FULL, *dims, 1)) == []"))
    assert all(same and exact and fits for same, exact, fits in got)


def test_the_matrices_calls_take_no_such_flag():
    from paper_1904_04956_amd import binding as bl
    for call in (lambda: bl.muon_matrices_step(4096, None, 4096, None, 1, 4, 4, 1, 0.1, 0.0, 0.0, bl.MUON_FULL, 4096, 1 << 30, 0),
                 lambda: bl.muon_adapters_step(4096, None, 4096, None, 4096, 1, 1, 4, 4, 1, 0.1, 0.0, 0.0, bl.MUON_FULL, 4096, 1 << 30, 0)):
        with pytest.raises(bl.BlstmError) as e:
            call()
        assert e.value.code == -2


@pytest.mark.gpu
@pytest.mark.parametrize("dims,flags", MODELS, ids=str)
def test_the_update_is_mode_0s(dims, flags):
    import torch
    from paper_1904_04956_amd import binding as bl
    g = torch.Generator(device="cuda:0").manual_seed(dims[1])
    out = []
    for mode, f in ((0, flags), (1, flags | bl.MUON_FULL)):
        ctx = bl.blstm_create(1, 1, *dims, mode)
        try:
            n = bl.blstm_param_count(ctx)
            if not out:
                start = [torch.randn(n, device="cuda:0", generator=g) * s for s in (0.1, 1e-3, 4e-3)]
            theta, grad, velocity = (t.clone() for t in start)
            shadow = torch.empty(n, dtype=torch.bfloat16, device="cuda:0")
            scratch = torch.full((bl.muon_scratch_bytes(ctx, f) + 4096,), 0x7F, dtype=torch.uint8, device="cuda:0")
            bl.muon_step(ctx, theta, shadow, grad, velocity, 0.02, 0.1, 0.9, 0.1, f, scratch, scratch.numel() - 4096)
            assert bool((scratch[-4096:] == 0x7F).all()) and torch.equal(shadow, theta.bfloat16())
            out.append((theta, velocity))
        finally:
            bl.blstm_destroy(ctx)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
