"""What runs around the tests: nothing that a test does not ask for, so that no test's mistakes are hidden by it."""


def test_no_fixture_of_every_test(request):
    assert request.fixturenames == ["request"]


def test_fills_end_for_one_test_only(request):
    for item in request.session.items:
        assert ("fills_end" in item.fixturenames) == item.nodeid.endswith("test_gpu_kv8.py::test_another_stream")
