"""smoke() runs every example, and with them every family of operators."""
import glob
import inspect
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_example_is_run():
    sys.path.insert(0, ROOT)
    import __graft_entry__
    source = inspect.getsource(__graft_entry__.smoke)
    examples = [os.path.splitext(os.path.basename(p))[0] for p in glob.glob(os.path.join(ROOT, "examples", "*.py"))]
    assert len(examples) >= 2 and all('"%s"' % name in source for name in examples)


def test_examples_call_every_family():
    text = "".join(open(p).read() for p in glob.glob(os.path.join(ROOT, "examples", "*.py")))
    for name in ("hla_conv", "hla_ssm", "hla_qk_norm", "hla_glr", "hla_block_norm", "hla_ffn"):
        assert name + "_forward(" in text, name
    for name in ("hla_conv", "hla_qk_norm", "hla_glr", "hla_block_norm", "hla_ffn"):
        assert name + "_backward(" in text, name
