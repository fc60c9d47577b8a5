"""The learning-rate schedule and the trainer's module come without PyTorch, the library's binding
alone; distillation loads it when it is called (CPU)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_schedule_does_not_load_torch():
    code = ("import sys; from paper_2410_05165_amd.align import cosine_lr, AlignTrainer, distill; "
            "assert cosine_lr(5, 10, 1.0, 5) == 1.0; assert 'torch' not in sys.modules")
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr
