"""Over how many workgroups attention splits its tiles, without a GPU: as many as the chip holds of the kernel that runs (256
compute units)."""
import pytest

from test_more_serving_abi import MORE_PRE, run  # noqa: F401

PLANS = """
def workgroups(call, *a, **kw):
    assert call(*a, **kw) == 0, lib.sats_last_error()
    n = [eval(l[2].replace("x", "*")) for l in log() if l[0] == "launch" and "join" not in l[1]]
    return n[0]
def plain(*a, form=0, **kw):
    return attend8(*a, form=form, **kw)
"""


# heads of dim, their form, the type of queries, and the workgroups of a compute unit
@pytest.mark.parametrize("dim,form,esz,held", [
    (64, 0, 2, 3), (80, 0, 2, 3), (96, 0, 2, 3), (96, 0, 4, 3), (112, 0, 2, 2), (128, 0, 4, 2), (256, 0, 2, 1),
    (64, 17, 2, 3), (64, 18, 4, 3), (80, 17, 2, 2), (96, 17, 2, 2), (96, 18, 2, 2), (96, 17, 4, 2), (128, 18, 2, 2), (256, 17, 2, 1)])
def test_a_split_fills_the_chip_once(run, dim, form, esz, held):  # noqa: F811
    """Eight sequences of so many keys that each part is shorter than what more workgroups are taken for: at most what is
    held at once, and more than half of it."""
    n = run(PLANS + f"print(json.dumps(workgroups(plain, 8, 8, 1, 3000, form={form}, esz={esz}, dim={dim})))")
    assert 256 * held // 2 < n <= 256 * held, n


@pytest.mark.parametrize("form", [0, 17, 18])
def test_phases_with_tiles_of_128_rows_hold_two(run, form):  # noqa: F811
    """... a compute unit, at every width up to 128: 16 single tokens on 4000 shared keys are split alike."""
    got = run(PLANS + f"""
print(json.dumps([workgroups(shared, 16, 16, 1, 6000, 1, 16, 4000, 2000, form={form}, dim=dim) for dim in (64, 80, 96, 128)]))""")
    assert len(set(got)) == 1, got


@pytest.mark.parametrize("form,esz", [(0, 2), (0, 4), (17, 2), (17, 4), (18, 2)])
def test_phases_of_tiles_of_16_rows_hold_three_up_to_64_dims(run, form, esz):  # noqa: F811
    """Four single tokens on a prefix, whose parts are long."""
    got = run(PLANS + f"""
print(json.dumps([workgroups(shared, 4, 4, 1, 30000, 1, 4, 28000, 2000, form={form}, esz={esz}, dim=dim) for dim in (64, 80, 96, 128)]))""")
    assert got[0] > got[1] and len(set(got[1:])) == 1, got
