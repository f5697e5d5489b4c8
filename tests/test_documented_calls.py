"""The calls that README.md shows take the arguments that it gives them (no GPU needed)."""
import ast
import inspect
import os
import re

import paper_2511_23225_amd as tw

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def shown_calls():
    """Each tw.name(...) of the text's blocks, parsed: from the name to the bracket that closes."""
    for block in re.findall(r"^```\w*\n(.*?)^```", open(README).read(), re.S | re.M):
        for m in re.finditer(r"\btw\.(\w+)\(", block):
            end, depth = m.end(), 1
            while depth:
                depth += {"(": 1, ")": -1}.get(block[end], 0)
                end += 1
            yield ast.parse(block[m.start():end], mode="eval").body


def test_calls_of_the_readme_bind():
    seen = set()
    for call in shown_calls():
        name = call.func.attr
        inspect.signature(getattr(tw, name)).bind(*call.args, **{k.arg: k.value for k in call.keywords})
        seen.add(name)
    assert {"tweo_rotary_freqs", "tweo_head_norm_rotary_fwd", "tweo_fp8_gated_fwd_bf16", "tweo_fp8_gated_bwd_bf16"} <= seen, seen
