// What the translation units of the tree operators share with the rest of the library.
#pragma once
// where calls without a context leave their error text (sjd_last_error(NULL))
char *sjd_call_error();
