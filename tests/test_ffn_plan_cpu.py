"""The gated block's planning on the host (no GPU)."""
from test_plan_cpu import run_host_program


def test_resident_clusters_are_a_devices_and_failures_are_not_kept():
    r = run_host_program("ffn_clusters")
    assert r.returncode == 0, r.stderr[-2000:]
    got = r.stdout.split()
    said = {k: int(v) for k, v in zip(got[::2], got[1::2])}
    assert said["failed"] < 1  # no clusters are counted on then
    assert (said["first"], said["again"], said["other"], said["back"]) == (10, 10, 11, 10)
    assert said["asked"] == 3  # the failure, and once a device


def test_a_joint_launch_deals_every_tile_once():
    r = run_host_program("ffn_deal")
    assert r.returncode == 0 and "bad 0" in r.stdout, r.stdout[-2000:]
    assert int(r.stdout.split("dealt ")[1].split(",")[0]) > 20000


def test_two_row_tiles_where_they_leave_every_sm_two_ctas():
    r = run_host_program("matvec_rows")
    assert r.returncode == 0, r.stderr[-2000:]
    got = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert got == [(s, 2 * 32 * s) for s in (100, 148, 152, 160)]
