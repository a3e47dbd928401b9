"""The timed steps of the benchmark follow its warm-up steps at once: 40 ms of anything else in between leave the GPU idle, and the steps after
that are slower by four per cent (4,000 events a step) to ten (200)."""
import ast
import inspect


def test_nothing_between_warm_up_and_clock_but_a_wait():
    import bench
    tree = ast.parse(inspect.getsource(bench.run_config))
    at = {}
    for n in ast.walk(tree):
        if isinstance(n, ast.Call):
            at.setdefault(ast.unparse(n), []).append(n.lineno)
    (warm,), (timed,) = at["run_steps(0, args.warmup)"], at["run_steps(args.warmup, args.warmup + args.steps)"]
    (collect,), (off,), (on,) = at["gc.collect()"], at["gc.disable()"], at["gc.enable()"]
    assert collect < off < warm < timed < on
    between = [k for k, lines in at.items() for line in lines if warm < line < timed]
    assert all(k in ("torch.cuda.synchronize()", "time.perf_counter()") or k.startswith("ctx.tgnn_profile_") for k in between), between
