"""The order of calls that README shows: what is stored on a side stream is joined before anything else touches the cache."""
import ast

from readme_check import example


def calls(tree):
    got = [(n.lineno, f"{n.func.value.id}.{n.func.attr}") for n in ast.walk(tree)
           if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute) and isinstance(n.func.value, ast.Name)]
    return [name for _, name in sorted(got)]


def test_stored_rows_are_joined_before_the_cache_is_used():
    names = calls(ast.parse(example()))
    run, join = names.index("path.run_layer"), names.index("path.join")
    assert names.index("path.store_into") < run < join
    assert all(not n.startswith("cache.") for n in names[run:join])
    assert join < names.index("cache.fork") < names.index("cache.append") < names.index("cache.plan") < names.index("cache.attend")
