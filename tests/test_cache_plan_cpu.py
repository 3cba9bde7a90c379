"""The packed cache's and the attention's index arithmetic on the host (no GPU)."""
from test_plan_cpu import run_host_program


def test_every_step_is_one_ctas_and_every_row_lies_in_the_cache():
    r = run_host_program("cache_walk")
    assert r.returncode == 0 and "bad 0" in r.stdout, (r.stdout + r.stderr)[-2000:]
    assert int(r.stdout.split("cases ")[1].split(",")[0]) > 4000
