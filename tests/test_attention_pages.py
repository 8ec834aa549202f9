"""Every kernel of the attention that the library's rule can choose, by that rule compiled here, is taken by a case of the GPU tests: each form (rows and waves to a workgroup)
for either head_dim, for steps of one page and of several, with keys that are split and that are not, into few or many splits, which are joined differently.
"""
import itertools

from test_attention_forms import ask  # noqa: F401 (a fixture)
import test_gpu_attention_forms as forms
import test_gpu_attention_pages as pages

STEP = 64       # keys


def kernel(head_dim, page, told):
    """(rows, waves, head_dim, a step in one page or not, 0: not split, 1: few splits, joined by the threads of a row, 2: by several groups of them)"""
    rows, waves, splits = told
    return rows, waves, head_dim, page >= STEP, 0 if splits == 1 else 1 if splits <= 256 // (head_dim // 4) else 2


def test_every_kernel_that_can_be_chosen_is_taken(ask):  # noqa: F811
    taken = set()
    for module, padding in ((forms, 5), (pages, pages.PADDING)):
        for heads, group, dim, page, window, plan in module.CASES.values():
            longest = (max((n + page - 1) // page for _, n in plan) + 1) * page
            (told,) = ask([(heads, dim, page, len(plan), heads * group, sum(n for n, _ in plan) + padding, window, longest)])
            taken.add(kernel(dim, page, told))
    calls = [(heads, dim, page, count, heads * group, rows, window, longest) for heads, dim, page, count, group, rows, window, longest in itertools.product(
        (1, 2, 3, 8, 12), (64, 128), (16, 32, 64, 128), (1, 2, 24, 48, 70), (1, 4, 8, 17), (1, 2, 24, 48, 70, 200, 360, 1000, 2500, 5000, 20000), (0, 300, 3000),
        (100, 900, 2000, 5000, 9800, 13000, 40000, 130000))]
    chosen = {}
    for call, told in zip(calls, ask(calls)):
        chosen.setdefault(kernel(call[1], call[2], told), call)
    assert not {k: c for k, c in chosen.items() if k not in taken}
    # what the launch has of them
    for dim, wide in itertools.product((64, 128), (False, True)):
        for rows, waves in ((16, 8), (16, 4), (32, 4), (128, 4)):
            assert {split for *k, split in chosen if k == [rows, waves, dim, wide]}, (rows, waves, dim, wide)
    assert {k[:4] for k in chosen if k[0] == 256} == {(256, 8, 128, True)}
