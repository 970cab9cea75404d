"""The format switch in threads whose calls overlap, nested, and entered again: every thread has its own format, and has the one
from before back when the block ends (no GPU)."""
import contextvars
import threading

import pytest

from paper_2509_26092_gb300 import dbl as D


def overlapping(first_work, second_work):
    """Two threads inside at once, the first in the first out; (what each raised, its format inside, its format after) of both."""
    entered, inside, left = threading.Event(), threading.Event(), threading.Event()
    seen = [None, None]

    def first():
        def body():
            entered.set()
            assert inside.wait(30)
            return D.current_precision()
        run(0, first_work, body)
        left.set()

    def second():
        assert entered.wait(30)

        def body():
            inside.set()
            assert left.wait(30)
            return D.current_precision()
        run(1, second_work, body)

    def run(i, work, body):
        error = within = None
        try:
            within = work(body)
        except Exception as e:  # reported by the test
            error = e
        seen[i] = (error, within, D.current_precision())

    threads = [threading.Thread(target=t) for t in (first, second)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    return seen


def test_a_decorated_function_in_two_threads():
    work = D.precision("f16")(lambda body: body())
    assert overlapping(work, work) == [(None, "f16", "bf16")] * 2
    assert D.current_precision() == "bf16"


def test_one_object_in_two_threads():
    fmt = D.precision("f16")

    def work(body):
        with fmt:
            return body()
    assert overlapping(work, work) == [(None, "f16", "bf16")] * 2
    assert D.current_precision() == "bf16"


def test_formats_of_two_threads_do_not_meet():
    works = [D.precision(p)(lambda body: body()) for p in ("f16", "bf16")]
    assert overlapping(*works) == [(None, "f16", "bf16"), (None, "bf16", "bf16")]


def test_nested_entered_again_and_left_by_an_exception():
    f16, bf16 = D.precision("f16"), D.precision("bf16")
    with f16:
        with bf16:
            with f16, f16:
                assert D.current_precision() == "f16"
            assert D.current_precision() == "bf16"
        assert D.current_precision() == "f16"
    assert D.current_precision() == "bf16"

    @f16
    def down(n):
        with bf16:
            assert D.current_precision() == "bf16"
        return D.current_precision() if n == 0 else down(n - 1)
    assert down(3) == "f16"
    with pytest.raises(KeyError):
        with f16:
            raise KeyError
    assert D.current_precision() == "bf16"


def test_a_copied_context_has_the_format_of_its_copy():
    """As a task started inside a block has it: what it enters and leaves does not reach the block's own context."""
    fmt = D.precision("f16")

    def task():
        before = D.current_precision()
        with D.precision("bf16"):
            within = D.current_precision()
        with fmt:
            pass
        return before, within, D.current_precision()
    with fmt:
        assert contextvars.copy_context().run(task) == ("f16", "bf16", "f16")
        assert D.current_precision() == "f16"
    assert D.current_precision() == "bf16"


def test_a_block_is_left_where_it_was_entered():
    """Elsewhere it is refused, and changes neither format."""
    fmt, other = D.precision("f16"), contextvars.Context()
    other.run(fmt.__enter__)
    with pytest.raises(ValueError):
        fmt.__exit__(None, None, None)
    assert D.current_precision() == "bf16" and other.run(D.current_precision) == "f16"
    with pytest.raises(ValueError), D.precision("bf16"):
        fmt.__exit__(None, None, None)
    other.run(fmt.__exit__, None, None, None)
    assert other.run(D.current_precision) == "bf16"


def test_blocks_that_do_not_nest():
    """As of two generators, the first of which is closed first: the other's block stays open."""
    def block(p):
        with D.precision(p):
            while True:
                yield D.current_precision()
    one, two = block("f16"), block("f16")
    assert next(one) == next(two) == "f16"
    one.close()
    assert D.current_precision() == next(two) == "f16"
    two.close()
    assert D.current_precision() == "bf16"
