"""Small programs that use the library as a network would."""
